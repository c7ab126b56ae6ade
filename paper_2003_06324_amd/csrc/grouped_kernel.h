// The experts' products: C(i,:) = A(row(i),:) * B_e, rows of a group after one another.
#pragma once
#include "routed_ring.h"
#include "routed_tile.h"

namespace gemm_gfx950 {

struct GroupedArgs {
    const void *A, *B;
    void *C;
    const int32_t *offsets, *row_map;
    int64_t lda, ldb, ldc, strideB;
    int groups, rows, a_rows, N, K, tiles_n;
};

// workgroups of a launch: as many tiles as there can be, whatever the groups' sizes
static inline int64_t grouped_grid(int64_t groups, int64_t rows, int64_t BM, int64_t tiles_n)
{
    return 8 * ceil_div((rows / BM + (groups < rows ? groups : rows)) * tiles_n, 8);
}

template <typename T, typename TC, int BM, int BN, int WM, int WN, int NST, bool BKC>
__global__ __launch_bounds__(WM *WN * 64) void grouped_kernel(const GroupedArgs p)
{
    typedef TileLoop<T, BM, BN, WM, WN, NST, true, BKC> Loop;
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    GroupTile g;
    if (!group_tile<BM>(p.offsets, p.groups, p.rows, p.tiles_n, lane, g)) return;
    const int m0 = g.tile_m * BM, n0 = g.tile_n * BN;
    const int n = (p.K + Loop::BK - 1) / Loop::BK, krem = p.K - (n - 1) * Loop::BK;

    RowsLoader<T, BM, Loop::NW> la;
    typename Loop::LoaderB lb;
    la.init_rows((const T *)p.A, p.lda, p.a_rows, p.row_map, g.lo, g.hi, m0, p.K, wave, lane);
    lb.init((const T *)p.B + (int64_t)g.group * p.strideB, p.ldb, n0, p.N, p.K, 0, wave, lane);
    auto at = [&](int h) {
        if (h > 0) {
            la.advance();
            lb.advance();
        }
        la.exact_range();
        lb.exact_range();
        if (h == n - 1 && krem < Loop::BK) {
            la.ragged_slab(krem, wave, lane);
            lb.ragged_slab(krem, wave, lane);
        }
    };
    float16_t acc[Loop::FM][Loop::FN];
    Loop::zero(acc);
    Loop::run(la, lb, at, n, krem, lds, acc, wave, lane);
    store_rows<TC, BM, BN, WM, WN, Loop::LDS_BYTES>(acc, lds, (TC *)p.C + (int64_t)(g.lo + m0) * p.ldc + n0, p.ldc, g.hi - g.lo - m0, p.N - n0, wave, lane);
}

// Large tiles, on the operand ring.
template <typename T, typename TC, int BM, int BN, bool BKC>
__global__ __launch_bounds__(256) void grouped_ring_kernel(const GroupedArgs p)
{
    typedef RingLoop<T, BM, BN, 2, 2, true, BKC> Loop;
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    GroupTile g;
    if (!group_tile<BM>(p.offsets, p.groups, p.rows, p.tiles_n, lane, g)) return;
    const int m0 = g.tile_m * BM, n0 = g.tile_n * BN;
    const int n = (p.K + Loop::BK - 1) / Loop::BK, krem = p.K - (n - 1) * Loop::BK;
    RingRowsLoader<T, BM, 4> la;
    RingLoader<T, BN, 4, BKC> lb;
    const T *const B = (const T *)p.B + (int64_t)g.group * p.strideB;
    la.init_rows((const T *)p.A, p.lda, p.a_rows, p.row_map, g.lo, g.hi, m0, p.K, wave, lane);
    lb.init(B, p.ldb, n0, p.N, wave, lane);
    const bool checked = krem < Loop::BK || lb.reaches_end(n0, p.N);
    float16_t acc[Loop::FM][Loop::FN];
    Loop::run(la, lb, la.end, DirectLoader<T, BN, 4, BKC>::end_of(B, p.ldb, p.N, p.K), checked, n, krem, lds, acc, wave, lane);
    store_rows<TC, BM, BN, 2, 2, Loop::LDS_BYTES>(acc, lds, (TC *)p.C + (int64_t)(g.lo + m0) * p.ldc + n0, p.ldc, g.hi - g.lo - m0, p.N - n0, wave, lane);
}

// The same through registers: any alignment, any leading dimension.
template <typename T, typename TC, int BM, int BN, bool BKC>
__global__ __launch_bounds__(256) void grouped_any_kernel(const GroupedArgs p)
{
    typedef TileLoop<T, BM, BN, 2, 2, 2, true, BKC> Loop;
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    GroupTile g;
    if (!group_tile<BM>(p.offsets, p.groups, p.rows, p.tiles_n, lane, g)) return;
    const int m0 = g.tile_m * BM, n0 = g.tile_n * BN;

    const T *const A = (const T *)p.A, *const B = (const T *)p.B + (int64_t)g.group * p.strideB;
    auto row_a = [&](int r) -> const T * {
        const int i = g.lo + m0 + r;
        if (i >= g.hi) return nullptr;
        const int row = p.row_map != nullptr ? p.row_map[i] : i;
        return row >= 0 && row < p.a_rows ? A + (int64_t)row * p.lda : nullptr;
    };
    auto row_b = [&](int r) -> const T * {  // column n0 + r of B, or its k-row r
        if (BKC) return n0 + r < p.N ? B + (int64_t)(n0 + r) * p.ldb : nullptr;
        return r < p.K ? B + (int64_t)r * p.ldb : nullptr;
    };
    GranuleLoader<T, BM, Loop::NT, true> la[GRANULE_DEPTH];
    GranuleLoader<T, BN, Loop::NT, BKC> lb[GRANULE_DEPTH];
    float16_t acc[Loop::FM][Loop::FN];
    Loop::zero(acc);
    auto fetch = [&](auto set, int k0) {
        la[set].fetch(row_a, 0, p.K, k0, tid);
        lb[set].fetch(row_b, n0, BKC ? p.K : p.N, k0, tid);
    };
    auto store = [&](auto set, int stage) {
        la[set].store(lds + stage, tid);
        lb[set].store(lds + stage + Loop::A_BYTES, tid);
    };
    granule_loop<Loop>(fetch, store, 0, p.K, lds, acc, wave, lane);
    store_rows<TC, BM, BN, 2, 2, Loop::LDS_BYTES>(acc, lds, (TC *)p.C + (int64_t)(g.lo + m0) * p.ldc + n0, p.ldc, g.hi - g.lo - m0, p.N - n0, wave, lane);
}

}  // namespace gemm_gfx950
