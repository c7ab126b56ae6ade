// Low-rank additions beside a shared projection: C(i,:) = A(i,:) B + scale_a (A(i,:) down_a) up_a, a = adapter_of[i].
//
// Two launches.  The first computes T(i,:) = scale_a A(i,:) down_a, rows x rank, in binary32, K cut into slices where the rows
// are few (the slices' sums lie one behind the other, and who reads T adds them up in slice order).  The second is the shared
// product, whose tiles, when their K loop is done, multiply their rows of T with the up matrices of the adapters that
// the tile has.  T is cut into 16-bit parts for the matrix instructions (two of binary16, three of bfloat16, relative to
// the row's largest, so that nothing overflows): what is lost of it is below 2^-22 of the row's largest element.
#pragma once
#include "gemm_small_kernel.h"
#include "routed_tile.h"

namespace gemm_gfx950 {

struct AdaptersArgs {
    const void *A, *B, *down, *up;
    void *C;
    const int32_t *adapter_of;
    const float *scales;
    float *t;               // [t_splits][rows][t_pitch]
    int64_t lda, ldb, ldc, ld_down, stride_down, ld_up, stride_up;
    int rows, N, K, adapters, rank, t_pitch, t_splits, t_k;  // t_k: k of a slice of T
    int up_kc;              // up is rank-contiguous (column-major)
    int tiles_m, tiles_n;
    Divisor by_band, by_last_rows;
};

__device__ __forceinline__ int adapter_at(const AdaptersArgs &p, int row)
{
    if (p.adapters == 0 || row >= p.rows) return -1;  // (without adapters there need not be any numbers)
    const int a = p.adapter_of[row];
    return a >= 0 && a < p.adapters ? a : -1;
}

constexpr int DOWN_ROWS = 32, DOWN_WAVES = 4;

// ---------------------------------------------------------------------------
// T: a workgroup takes 32 rows and a slice of K (blockIdx.x), and of the adapters that its rows have those whose number is blockIdx.y modulo
// gridDim.y; its waves share out the slice's k-groups and their sums meet in LDS, in wave order.  KC: down is K-contiguous.
// ---------------------------------------------------------------------------
template <typename T, bool KC> __global__ __launch_bounds__(DOWN_WAVES * 64) void adapters_down_kernel(const AdaptersArgs p)
{
    constexpr int KG = Elem<T>::KG, EPL = KG / 2;
    typedef typename Frag<T>::type frag_t;
    __shared__ float part[DOWN_WAVES][32][33];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int slice = (int)blockIdx.x % p.t_splits, m0 = (int)blockIdx.x / p.t_splits * DOWN_ROWS;
    const int k0 = slice * p.t_k, k1 = k0 + p.t_k < p.K ? k0 + p.t_k : p.K;
    const int id = adapter_at(p, m0 + (lane & 31));
    const int row = m0 + (lane & 31) < p.rows ? m0 + (lane & 31) : p.rows - 1;
    const uint32_t turn = blockIdx.y, turns = gridDim.y;
    int a = -1;
    for (;;) {
        const uint32_t next = umin_over<64>(id > a && (uint32_t)id % turns == turn ? (uint32_t)id : 0xffffffffu);
        if (next == 0xffffffffu) break;
        a = __builtin_amdgcn_readfirstlane((int)next);
        const float scale = p.scales != nullptr ? p.scales[a] : 1.0f;
        const T *const down = (const T *)p.down + (int64_t)a * p.stride_down;
        for (int q0 = 0; q0 < p.rank; q0 += 32) {
            const int q = q0 + (lane & 31) < p.rank ? q0 + (lane & 31) : p.rank - 1;
            float16_t acc;
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
            auto group = [&](int k, bool full) {
                const int kl = k + (lane >> 5) * EPL;
                const frag_t fa = small_fragment<T, true>((const T *)p.A, p.lda, row, kl, p.K, full);
                const frag_t fb = small_fragment<T, KC>(down, p.ld_down, q, kl, p.K, full);
                mma(acc, fa, fb);
            };
            int k = k0 + wave * KG;
#pragma unroll 4
            for (; k + KG <= k1; k += DOWN_WAVES * KG) group(k, true);
            if (k < k1) group(k, false);
#pragma unroll
            for (int r = 0; r < 16; ++r) part[wave][8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)][lane & 31] = acc[r];
            __syncthreads();
            const int here = q0 + (tid & 31);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = i * 8 + (tid >> 5);
                float sum = part[0][r][tid & 31];
#pragma unroll
                for (int w = 1; w < DOWN_WAVES; ++w) sum += part[w][r][tid & 31];
                if (here < p.rank && adapter_at(p, m0 + r) == a) p.t[((int64_t)slice * p.rows + m0 + r) * p.t_pitch + here] = scale * sum;
            }
            __syncthreads();
        }
    }
}

// Number of 16-bit parts of a binary32 number
template <typename T> struct Parts;
template <> struct Parts<float> { static constexpr int N = 1; };
template <> struct Parts<_Float16> { static constexpr int N = 2; };
template <> struct Parts<__bf16> { static constexpr int N = 3; };

// ---------------------------------------------------------------------------
// The additions of a tile of the shared product, added to its accumulators.  lds: the K loop's stages, drained of loads.
// ---------------------------------------------------------------------------
template <typename T, typename Loop, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void add_adapters(const AdaptersArgs &p, GEMM_LDS(char) * lds, float16_t (&acc)[Loop::FM][Loop::FN], int m0, int n0, int tid, int wave,
                                             int lane)
{
    constexpr int NT = Loop::NT, EPC = Elem<T>::EPC, BK = Elem<T>::BK, KG = Elem<T>::KG, NP = Parts<T>::N;
    constexpr int ITERS = BM * GPR / NT, FM = Loop::FM, FN = Loop::FN;
    static_assert(NP * Loop::A_BYTES + Loop::B_BYTES <= Loop::LDS_BYTES, "the parts' images do not fit the stages");
    typedef typename Frag<T>::type frag_t;
    if (p.adapters == 0) return;
    __shared__ int ids[BM];
    __shared__ float row_scale[BM];
    const T *const up0 = (const T *)p.up;
    __syncthreads();  // every wave has read its last operands
    for (int r = tid; r < BM; r += NT) ids[r] = adapter_at(p, m0 + r);
    __syncthreads();
    auto t_value = [&](int row, int q) {
        const float *t = p.t + (int64_t)row * p.t_pitch + q;
        float sum = t[0];
        for (int s = 1; s < p.t_splits; ++s) sum += t[(int64_t)s * p.rows * p.t_pitch];
        return sum;
    };
    // a row's power of two: its largest element lies in [1, 2) without it
    float factor[ITERS];
#pragma unroll
    for (int i = 0; i < ITERS; ++i) {
        const int r = (tid + i * NT) / GPR, g = tid % GPR;
        factor[i] = 1.0f;
        if (sizeof(T) == 4) continue;
        float m = 0.0f;
        if (ids[r] >= 0)
            for (int q = g; q < p.rank; q += GPR) m = fmaxf(m, fabsf(t_value(m0 + r, q)));
#pragma unroll
        for (int s = 1; s < GPR; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
        int e = 0;
        if (m > 0.0f && m < INFINITY) e = ilogbf(m);
        // (2^-e itself can be out of range; 126 is the most that is taken off, and what is left then is below 2^-22 all the same)
        e = e < -126 ? -126 : e;
        factor[i] = ldexpf(1.0f, -e);
        if (g == 0) row_scale[r] = ldexpf(1.0f, e);
    }
    // Rows of other adapters take part in a product and are not taken over: masked to zeros they would meet this adapter's matrix
    // all the same, and a NaN or an infinity in it would reach them.
    const int wm = wave / WN, wn = wave % WN;
    int a = -1;
    bool t_there = false;  // the images hold all of T's parts
    for (;;) {
        uint32_t next = 0xffffffffu;
#pragma unroll
        for (int r = lane; r < BM; r += 64) {
            const int id = ids[r];
            if (id > a && (uint32_t)id < next) next = (uint32_t)id;
        }
        next = umin_over<64>(next);
        if (next == 0xffffffffu) break;
        a = __builtin_amdgcn_readfirstlane((int)next);
        const T *const up = up0 + (int64_t)a * p.stride_up;
        float16_t add[FM][FN];
        Loop::zero(add);
        for (int q0 = 0; q0 < p.rank; q0 += BK) {
#pragma unroll
            for (int i = 0; i < ITERS; ++i) {
                if (t_there) break;
                const int x = tid + i * NT, r = x / GPR, g = x % GPR;
                T v[NP][EPC];
#pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    const int q = q0 + g * EPC + e;
                    float left = ids[r] >= 0 && q < p.rank ? t_value(m0 + r, q) * factor[i] : 0.0f;
#pragma unroll
                    for (int n = 0; n < NP; ++n) {
                        v[n][e] = rounded<T>(left);
                        const float part = (float)v[n][e];
                        left = fabsf(part) < INFINITY ? left - part : 0.0f;
                    }
                }
#pragma unroll
                for (int n = 0; n < NP; ++n) {
                    uint4_t w;
                    __builtin_memcpy(&w, v[n], 16);
                    *(GEMM_LDS(uint4_t) *)(lds + n * Loop::A_BYTES + r * RBK + ((g ^ swz_kc(r)) << 4)) = w;
                }
            }
            t_there = p.rank <= BK;
            for (int x = tid; x < BN * GPR; x += NT) {
                const int c = x / GPR, g = x % GPR;
                T v[EPC];
#pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    const int q = q0 + g * EPC + e;
                    const bool there = q < p.rank && n0 + c < p.N;
                    v[e] = there ? up[p.up_kc ? (int64_t)(n0 + c) * p.ld_up + q : (int64_t)q * p.ld_up + n0 + c] : (T)0.0f;
                }
                uint4_t w;
                __builtin_memcpy(&w, v, 16);
                *(GEMM_LDS(uint4_t) *)(lds + NP * Loop::A_BYTES + c * RBK + ((g ^ swz_kc(c)) << 4)) = w;
            }
            __syncthreads();
#pragma unroll
            for (int kg = 0; kg < KGS; ++kg) {
                if (q0 + kg * KG >= p.rank) break;
                frag_t fb[FN];
#pragma unroll
                for (int j = 0; j < FN; ++j) fb[j] = Fetch<T, BN, true>::get(lds + NP * Loop::A_BYTES, wn * Loop::TN + j * 32, kg, lane);
#pragma unroll
                for (int n = NP - 1; n >= 0; --n)  // the small parts first
#pragma unroll
                    for (int i = 0; i < FM; ++i) {
                        const frag_t fa = Fetch<T, BM, true>::get(lds + n * Loop::A_BYTES, wm * Loop::TM + i * 32, kg, lane);
#pragma unroll
                        for (int j = 0; j < FN; ++j) mma(add[i][j], fa, fb[j]);
                    }
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int row = wm * Loop::TM + i * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
                const bool mine = ids[row] == a;
                const float f = sizeof(T) == 4 ? 1.0f : row_scale[row];
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j][r] = mine ? fmaf(add[i][j][r], f, acc[i][j][r]) : acc[i][j][r];
            }
    }
}

// tile of this workgroup: every XCD one contiguous run, in bands of tile rows
__device__ __forceinline__ bool adapters_tile(const AdaptersArgs &p, int &tile_m, int &tile_n)
{
    const int tiles = p.tiles_m * p.tiles_n, per_xcd = (tiles + 7) >> 3, i = blockIdx.x >> 3, w = (int)(blockIdx.x & 7) * per_xcd + i;
    if (i >= per_xcd || w >= tiles) return false;
    tile_at(p.tiles_m, p.tiles_n, p.by_band, p.by_last_rows, w, tile_m, tile_n);
    return true;
}

template <typename T, typename TC, int BM, int BN, int WM, int WN, int NST, bool BKC>
__global__ __launch_bounds__(WM *WN * 64) void adapters_kernel(const AdaptersArgs p)
{
    typedef TileLoop<T, BM, BN, WM, WN, NST, true, BKC> Loop;
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tile_m, tile_n;
    if (!adapters_tile(p, tile_m, tile_n)) return;
    const int m0 = tile_m * BM, n0 = tile_n * BN;
    const int n = (p.K + Loop::BK - 1) / Loop::BK, krem = p.K - (n - 1) * Loop::BK;
    typename Loop::LoaderA la;
    typename Loop::LoaderB lb;
    la.init((const T *)p.A, p.lda, m0, p.rows, p.K, 0, wave, lane);
    lb.init((const T *)p.B, p.ldb, n0, p.N, p.K, 0, wave, lane);
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
    add_adapters<T, Loop, BM, BN, WM, WN>(p, lds, acc, m0, n0, tid, wave, lane);
    store_rows<TC, BM, BN, WM, WN, Loop::LDS_BYTES>(acc, lds, (TC *)p.C + (int64_t)m0 * p.ldc + n0, p.ldc, p.rows - m0, p.N - n0, wave, lane);
}

// The same through registers: any alignment, any leading dimension.
template <typename T, typename TC, int BM, int BN, bool BKC>
__global__ __launch_bounds__(256) void adapters_any_kernel(const AdaptersArgs p)
{
    typedef TileLoop<T, BM, BN, 2, 2, 2, true, BKC> Loop;
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tile_m, tile_n;
    if (!adapters_tile(p, tile_m, tile_n)) return;
    const int m0 = tile_m * BM, n0 = tile_n * BN;
    const T *const A = (const T *)p.A, *const B = (const T *)p.B;
    auto row_a = [&](int r) -> const T * { return m0 + r < p.rows ? A + (int64_t)(m0 + r) * p.lda : nullptr; };
    auto row_b = [&](int r) -> const T * {
        if (BKC) return n0 + r < p.N ? B + (int64_t)(n0 + r) * p.ldb : nullptr;
        return r < p.K ? B + (int64_t)r * p.ldb : nullptr;
    };
    GranuleLoader<T, BM, Loop::NT, true> la;
    GranuleLoader<T, BN, Loop::NT, BKC> lb;
    float16_t acc[Loop::FM][Loop::FN];
    Loop::zero(acc);
    auto fetch = [&](int k0) {
        la.fetch(row_a, 0, p.K, k0, tid);
        lb.fetch(row_b, n0, BKC ? p.K : p.N, k0, tid);
    };
    if (p.K > 0) fetch(0);
    int stage = 0;
    for (int k0 = 0; k0 < p.K; k0 += Loop::BK) {
        la.store(lds + stage, tid);
        lb.store(lds + stage + Loop::A_BYTES, tid);
        if (k0 + Loop::BK < p.K) fetch(k0 + Loop::BK);
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
        barrier_keep_loads();
        Loop::multiply(lds + stage, lds + stage + Loop::A_BYTES, acc, wave, lane);
        stage = Loop::STAGE - stage;
    }
    add_adapters<T, Loop, BM, BN, 2, 2>(p, lds, acc, m0, n0, tid, wave, lane);
    store_rows<TC, BM, BN, 2, 2, Loop::LDS_BYTES>(acc, lds, (TC *)p.C + (int64_t)m0 * p.ldc + n0, p.ldc, p.rows - m0, p.N - n0, wave, lane);
}

}  // namespace gemm_gfx950
