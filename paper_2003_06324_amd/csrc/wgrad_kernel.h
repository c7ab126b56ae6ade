// Gradients of the experts' matrices: C_e = sum over the group's rows of X(i,:)^T * Y(i,:).
#pragma once
#include "routed_ring.h"
#include "routed_tile.h"

namespace gemm_gfx950 {

struct WgradArgs {
    const void *X, *Y;   // rows of C are columns of X, columns of C columns of Y
    void *C;
    const int32_t *offsets, *map_x, *map_y;  // (one of the maps at most)
    int64_t ldx, ldy, ldc, strideC;
    int groups, rows, x_rows, y_rows, M, N, tiles_m, tiles_n;
    int stream;  // C is stored past the L2
    int run;     // wgrad_run()
};

// Direct loads of an operand whose k-rows are a group's rows.  Without a map its base moves from slab to slab.  With one the lanes' offsets
// are set anew for every slab: a wave's rows are neighbours in the map, so their numbers are scalar loads, one slab ahead, and
// cost the vector unit a selection and an addition for each load.
template <typename T, int R, int NW, bool MAPPED> struct RingKRowsLoader : RingLoader<T, R, NW, false> {
    typedef RingLoader<T, R, NW, false> base_t;
    static constexpr int CPR = base_t::CPR, PER_WAVE = base_t::PER_WAVE, BK = base_t::BK, EPC = base_t::EPC;
    static constexpr int RPL = 64 / CPR, ROWS = PER_WAVE * RPL;  // k-rows of a load, of a wave
    static_assert(64 % CPR == 0 && ROWS * NW == BK && ROWS % 4 == 0, "whole k-rows");
    typedef const __attribute__((address_space(4))) uint32_t *numbers_t;
    uint64_t end;
    const int32_t *map;   // the whole map
    int at, rows;         // entry of it that `next` begins with, and their number
    uint32_t there, ldb;  // rows of the operand, bytes between them (all of them below 2^31)
    uint32_t next[MAPPED ? ROWS : 1];
    uint32_t col[2];      // the lane's place in its row, of the two swizzles that its loads have

    static constexpr int swizzle_of(int i) { return RPL == 4 ? 0 : (sizeof(T) == 2 ? i & 1 : (i * RPL >> 2) & 1); }

    // map_, rows_: the map of all groups, and how many entries it has (at least BK)
    __device__ __forceinline__ void init_rows(const T *X, int64_t ld, int rows_there, const int32_t *map_, int rows_, int lo, int hi, int col0, int cols, int wave,
                                              int lane)
    {
        typedef DirectLoader<T, R, NW, false> ends_t;
        if constexpr (!MAPPED) {
            const T *const first = X + (int64_t)lo * ld;
            this->init(first, ld, col0, cols, wave, lane);
            end = hi > lo ? ends_t::end_of(first, ld, cols, hi - lo) : 0;
        } else {
            this->init(X, ld, col0, cols, wave, lane);
            there = (uint32_t)rows_there;
            end = there > 0 ? ends_t::end_of(X, ld, cols, rows_there) : 0;
            map = map_;
            rows = rows_;
            ldb = (uint32_t)(ld * (int64_t)sizeof(T));
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int i = x == 0 || RPL == 4 ? 0 : (sizeof(T) == 2 ? 1 : 4 / RPL);  // a load with that swizzle
                const int kk = i * RPL + lane / CPR;
                const int m = ((lane % CPR) ^ swz_mc<T, CPR>(kk)) * EPC;
                col[x] = (uint32_t)((col0 + m < cols ? m : 0) * (int)sizeof(T));
            }
            // any slab may hold the operand's last row: the range always ends with the operand (its base stays)
            base_t::last_slab(end, BK, wave, lane);
            at = lo + wave * ROWS;
            numbers();
            offsets(lane);
            at += BK;
            numbers();
        }
    }
    // Rows behind the group's last one are other groups', or, at the map's end, any: rows_until() sees to them.
    __device__ __forceinline__ void numbers()
    {
        const numbers_t m = (numbers_t)(uintptr_t)(map + (at < rows - ROWS ? at : rows - ROWS));
#pragma unroll
        for (int r = 0; r < ROWS; ++r) next[r] = m[r];
    }
    __device__ __forceinline__ void offsets(int lane)
    {
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) {
            uint32_t row[RPL];
#pragma unroll
            for (int x = 0; x < RPL; ++x) {
                // a number that names no row becomes the one behind the last, which the loads' range leaves out
                const uint32_t r = next[i * RPL + x];
                row[x] = (r < there ? r : there) * ldb;
            }
            uint32_t mine = row[0];
#pragma unroll
            for (int x = 1; x < RPL; ++x) mine = lane / CPR == x ? row[x] : mine;
            this->off[i] = mine + col[swizzle_of(i)];
        }
    }
    // The slab whose first row is entry `first` of the map has `count` rows: the others are zeros, and the window of numbers may have been
    // moved back from the map's end, so the lanes ask for theirs themselves.
    __device__ __forceinline__ void rows_until(int count, int first, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) {
            const int kk = wave * ROWS + i * RPL + lane / CPR;
            uint32_t r = there;
            if (kk < count) {
                r = (uint32_t)map[first + kk];
                r = r < there ? r : there;
            }
            this->off[i] = kk < count ? r * ldb + col[swizzle_of(i)] : NO_ROW;
        }
    }
    __device__ __forceinline__ void last_slab(uint64_t to, int krem, int wave, int lane)
    {
        if constexpr (!MAPPED) {
            base_t::last_slab(to, krem, wave, lane);
        } else if (krem < BK) {  // (offsets() has moved on already)
            rows_until(krem, at - BK - wave * ROWS, wave, lane);
        }
    }
    // The numbers for the next advance().  The fragments' reads are waited for first: with scalar loads on their way every wait of
    // either kind is one for all of them, and the next one is the barrier's, a k-group from here.
    __device__ __forceinline__ void prefetch()
    {
        if constexpr (MAPPED) {
            __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
            numbers();
        }
    }
    __device__ __forceinline__ void advance(bool more)
    {
        if constexpr (!MAPPED) {
            base_t::advance(more);
        } else if (more) {
            offsets(threadIdx.x & 63);
            at += BK;
        }
    }
};

// Tiles in a row that one XCD takes: they are neighbours in their matrix and share panels in its L2.  While all tiles run at once their order
// is no matter and an XCD gets one run of them.
constexpr int WGRAD_RUN = 8;
static inline int wgrad_run(int64_t tiles) { return tiles > 64 * WGRAD_RUN ? WGRAD_RUN : (int)ceil_div(tiles, 8); }
static inline int64_t wgrad_grid(int64_t tiles) { return ceil_div(tiles, 8 * wgrad_run(tiles)) * 8 * wgrad_run(tiles); }
// Tile of this workgroup.  A tile takes as long as its group has rows, so the longest are dealt first and the XCDs get runs of the same
// length in turn: what is left at the end is short.  (Groups are ordered 64 at a time.)
__device__ __forceinline__ bool wgrad_tile(const WgradArgs &p, int lane, int &group, int &tile_m, int &tile_n)
{
    const uint32_t per = (uint32_t)p.tiles_m * (uint32_t)p.tiles_n;
    const uint32_t run = (uint32_t)p.run, turn = blockIdx.x >> 3, runs = turn / run;
    const uint32_t t = (runs * 8 + (blockIdx.x & 7)) * run + (turn - runs * run);
    const uint32_t place = t / per, in = t - place * per;
    if (place >= (uint32_t)p.groups) return false;
    const int c = (int)(place & ~63u), n = p.groups - c < 64 ? p.groups - c : 64;
    int slabs = -1;
    if (lane < n) {
        const Span s = group_span(p.offsets, c + lane, p.rows);
        slabs = (s.hi - s.lo + 63) / 64;
    }
    const int key = slabs * 64 + (63 - lane);  // of equal ones the first comes first
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += __builtin_amdgcn_readlane(key, j) > key;
    group = c + __builtin_ctzll(__ballot(lane < n && rank == (int)(place & 63)));
    tile_n = __builtin_amdgcn_readfirstlane((int)(in / (uint32_t)p.tiles_m));
    tile_m = __builtin_amdgcn_readfirstlane((int)(in - (uint32_t)tile_n * (uint32_t)p.tiles_m));
    return true;
}

// MAPPED: 0 no map, 1 X's rows are gathered, 2 Y's
template <typename T, typename TC, int BM, int BN, int MAPPED>
__global__ __launch_bounds__(256) void wgrad_kernel(const WgradArgs p)
{
    typedef RingLoop<T, BM, BN, 2, 2, false, false> Loop;
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int group, tile_m, tile_n;
    if (!wgrad_tile(p, lane, group, tile_m, tile_n)) return;
    const Span s = group_span(p.offsets, group, p.rows);
    const int lo = __builtin_amdgcn_readfirstlane(s.lo), hi = __builtin_amdgcn_readfirstlane(s.hi);
    const int m0 = tile_m * BM, n0 = tile_n * BN, count = hi - lo;
    const int n = (count + Loop::BK - 1) / Loop::BK, krem = count - (n - 1) * Loop::BK;
    RingKRowsLoader<T, BM, 4, MAPPED == 1> lx;
    RingKRowsLoader<T, BN, 4, MAPPED == 2> ly;
    lx.init_rows((const T *)p.X, p.ldx, p.x_rows, p.map_x, p.rows, lo, hi, m0, p.M, wave, lane);
    ly.init_rows((const T *)p.Y, p.ldy, p.y_rows, p.map_y, p.rows, lo, hi, n0, p.N, wave, lane);
    const bool checked = krem < Loop::BK || lx.reaches_end(m0, p.M) || ly.reaches_end(n0, p.N);
    float16_t acc[Loop::FM][Loop::FN];
    Loop::run(lx, ly, lx.end, ly.end, checked, n, krem, lds, acc, wave, lane);
    store_rows<TC, BM, BN, 2, 2, Loop::LDS_BYTES>(acc, lds, (TC *)p.C + (int64_t)group * p.strideC + (int64_t)m0 * p.ldc + n0, p.ldc, p.M - m0, p.N - n0, wave, lane, p.stream != 0);
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
    if (!wgrad_tile(p, lane, group, tile_m, tile_n)) return;
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
    GranuleLoader<T, BM, Loop::NT, false> lx[GRANULE_DEPTH];
    GranuleLoader<T, BN, Loop::NT, false> ly[GRANULE_DEPTH];
    float16_t acc[Loop::FM][Loop::FN];
    Loop::zero(acc);
    auto fetch = [&](auto set, int k0) {
        lx[set].fetch(row_x, m0, p.M, k0, tid);
        ly[set].fetch(row_y, n0, p.N, k0, tid);
    };
    auto store = [&](auto set, int stage) {
        lx[set].store(lds + stage, tid);
        ly[set].store(lds + stage + Loop::A_BYTES, tid);
    };
    granule_loop<Loop>(fetch, store, 0, count, lds, acc, wave, lane);
    store_rows<TC, BM, BN, 2, 2, Loop::LDS_BYTES>(acc, lds, (TC *)p.C + (int64_t)group * p.strideC + (int64_t)m0 * p.ldc + n0, p.ldc, p.M - m0, p.N - n0, wave, lane, p.stream != 0);
}

}  // namespace gemm_gfx950
