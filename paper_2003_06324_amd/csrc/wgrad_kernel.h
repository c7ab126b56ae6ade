// Gradients of the experts' matrices: C_e = sum over the group's rows of X(i,:)^T * Y(i,:).
#pragma once
#include "routed_tile.h"

namespace gemm_gfx950 {

struct WgradArgs {
    const void *X, *Y;   // rows of C are columns of X, columns of C columns of Y
    void *C;
    const int32_t *offsets, *map_x, *map_y;  // (one of the maps at most)
    int64_t ldx, ldy, ldc, strideC;
    int groups, rows, x_rows, y_rows, M, N, tiles_m, tiles_n;
};

constexpr int MAP_WINDOW = 4096;  // row numbers of a group kept in LDS

// Direct loads of an operand whose k-rows are a group's rows.  Without a map its base moves from slab to slab; with one the lanes'
// offsets are set anew for every slab, from row numbers in LDS.
template <typename T, int R, int NW> struct KRowsLoader : StageLoader<T, R, NW, false> {
    typedef StageLoader<T, R, NW, false> base_t;
    __device__ __forceinline__ void init_rows(const T *X, int64_t ld, int there, bool mapped, int lo, int hi, int col0, int cols, int wave, int lane)
    {
        const int last = mapped ? there : (there < hi ? there : hi) - lo;  // rows from the origin on
        this->init(mapped ? X : X + (int64_t)lo * ld, ld, col0, cols, last > 0 ? last : 1, 0, wave, lane);
        if (last <= 0) this->no_rows();
    }
    __device__ __forceinline__ void no_rows() { this->end = 0; }
    // the range ends with the operand's rows, of which there may be none left (rows of the group behind A's last one)
    __device__ __forceinline__ void range()
    {
        const uint64_t base = ((uint64_t)(uint32_t)this->rsrc[1] << 32) | (uint32_t)this->rsrc[0];
        if (base >= this->end) this->no_range();
        else this->exact_range();
    }
    // slab from k-row k on; window: the row numbers in LDS, from a multiple of MAP_WINDOW
    __device__ __forceinline__ void gather(const GEMM_LDS(int) * window, int64_t ld, int there, int col0, int cols, int k, int count, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < base_t::PER_WAVE; ++i) {
            const int q = 64 * (wave * base_t::PER_WAVE + i) + lane;
            const int kk = q / base_t::CPR;
            const int m = ((q % base_t::CPR) ^ swz_mc<T, base_t::CPR>(kk)) * base_t::EPC;
            const int row = window[(k + kk) & (MAP_WINDOW - 1)];
            const uint32_t at = (uint32_t)row * (uint32_t)(ld * (int64_t)sizeof(T)) + (uint32_t)((col0 + m < cols ? m : 0) * (int)sizeof(T));
            this->off[i] = k + kk < count && row >= 0 && row < there ? at + base_t::LEAD - i % base_t::GROUP * 1024 : NO_ROW;
        }
    }
};

// tile of this workgroup: matrix by matrix, every XCD one contiguous run
__device__ __forceinline__ bool wgrad_tile(const WgradArgs &p, int &group, int &tile_m, int &tile_n)
{
    const uint32_t per = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n, tiles = per * (uint32_t)p.groups, per_xcd = (tiles + 7) / 8;
    const uint32_t i = blockIdx.x >> 3, w = (blockIdx.x & 7) * per_xcd + i;
    if (i >= per_xcd || w >= tiles) return false;
    group = (int)(w / per);
    const uint32_t in = w - (uint32_t)group * per;
    tile_n = (int)(in / (uint32_t)p.tiles_m);
    tile_m = (int)(in - (uint32_t)tile_n * (uint32_t)p.tiles_m);
    return true;
}

template <typename T, typename TC, int BM, int BN, int WM, int WN, int NST>
__global__ __launch_bounds__(WM *WN * 64) void wgrad_kernel(const WgradArgs p)
{
    typedef TileLoop<T, BM, BN, WM, WN, NST, false, false> Loop;
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    __shared__ int window_[MAP_WINDOW];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    GEMM_LDS(int) *window = (GEMM_LDS(int) *)window_;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int group, tile_m, tile_n;
    if (!wgrad_tile(p, group, tile_m, tile_n)) return;
    const Span s = group_span(p.offsets, group, p.rows);
    const int lo = __builtin_amdgcn_readfirstlane(s.lo), hi = __builtin_amdgcn_readfirstlane(s.hi);
    const int m0 = tile_m * BM, n0 = tile_n * BN, count = hi - lo;
    const int n = (count + Loop::BK - 1) / Loop::BK;
    const int32_t *const map = p.map_x != nullptr ? p.map_x : p.map_y;

    KRowsLoader<T, BM, Loop::NW> lx;
    KRowsLoader<T, BN, Loop::NW> ly;
    lx.init_rows((const T *)p.X, p.ldx, p.x_rows, p.map_x != nullptr, lo, hi, m0, p.M, wave, lane);
    ly.init_rows((const T *)p.Y, p.ldy, p.y_rows, p.map_y != nullptr, lo, hi, n0, p.N, wave, lane);
    auto at = [&](int h) {
        if (map != nullptr && h * Loop::BK % MAP_WINDOW == 0) {
            __syncthreads();  // the numbers before are done with
            for (int i = tid; i < MAP_WINDOW; i += Loop::NT) window[i] = h * Loop::BK + i < count ? map[lo + h * Loop::BK + i] : -1;
            __syncthreads();
        }
        if (p.map_x != nullptr) lx.gather(window, p.ldx, p.x_rows, m0, p.M, h * Loop::BK, count, wave, lane);
        else if (h > 0) lx.advance();
        if (p.map_y != nullptr) ly.gather(window, p.ldy, p.y_rows, n0, p.N, h * Loop::BK, count, wave, lane);
        else if (h > 0) ly.advance();
        lx.range();
        ly.range();
    };
    float16_t acc[Loop::FM][Loop::FN];
    Loop::zero(acc);
    Loop::run(lx, ly, at, n, Loop::BK, lds, acc, wave, lane);  // (rows past the last one are zeros)
    store_rows<TC, BM, BN, WM, WN, Loop::LDS_BYTES>(acc, lds, (TC *)p.C + (int64_t)group * p.strideC + (int64_t)m0 * p.ldc + n0, p.ldc, p.M - m0, p.N - n0, wave, lane);
}

// The same through registers: any alignment, any leading dimension.
template <typename T, typename TC, int BM, int BN>
__global__ __launch_bounds__(256) void wgrad_any_kernel(const WgradArgs p)
{
    typedef TileLoop<T, BM, BN, 2, 2, 2, false, false> Loop;
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int group, tile_m, tile_n;
    if (!wgrad_tile(p, group, tile_m, tile_n)) return;
    const Span s = group_span(p.offsets, group, p.rows);
    const int lo = __builtin_amdgcn_readfirstlane(s.lo), hi = __builtin_amdgcn_readfirstlane(s.hi);
    const int m0 = tile_m * BM, n0 = tile_n * BN, count = hi - lo;
    auto row_of = [&](const T *base, int64_t ld, const int32_t *map, int there, int k) -> const T * {
        if (k >= count) return nullptr;
        const int row = map != nullptr ? map[lo + k] : lo + k;
        return row >= 0 && row < there ? base + (int64_t)row * ld : nullptr;
    };
    auto row_x = [&](int k) { return row_of((const T *)p.X, p.ldx, p.map_x, p.x_rows, k); };
    auto row_y = [&](int k) { return row_of((const T *)p.Y, p.ldy, p.map_y, p.y_rows, k); };
    GranuleLoader<T, BM, Loop::NT, false> lx;
    GranuleLoader<T, BN, Loop::NT, false> ly;
    float16_t acc[Loop::FM][Loop::FN];
    Loop::zero(acc);
    auto fetch = [&](int k0) {
        lx.fetch(row_x, m0, p.M, k0, tid);
        ly.fetch(row_y, n0, p.N, k0, tid);
    };
    if (count > 0) fetch(0);
    int stage = 0;
    for (int k0 = 0; k0 < count; k0 += Loop::BK) {
        lx.store(lds + stage, tid);
        ly.store(lds + stage + Loop::A_BYTES, tid);
        if (k0 + Loop::BK < count) fetch(k0 + Loop::BK);
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
        barrier_keep_loads();
        Loop::multiply(lds + stage, lds + stage + Loop::A_BYTES, acc, wave, lane);
        stage = Loop::STAGE - stage;
    }
    store_rows<TC, BM, BN, 2, 2, Loop::LDS_BYTES>(acc, lds, (TC *)p.C + (int64_t)group * p.strideC + (int64_t)m0 * p.ldc + n0, p.ldc, p.M - m0, p.N - n0, wave, lane);
}

}  // namespace gemm_gfx950
