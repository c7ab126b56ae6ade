// Low-rank additions beside a shared projection: C(i,:) = A(i,:) B + scale_a (A(i,:) down_a) up_a, a = adapter_of[i].
//
// With T(i,:) = scale_a A(i,:) down_a, rows x rank, held in binary32:
//   few rows:  one launch computes T and the shared product, both in slices of K (a few rows would not give every CU
//              work otherwise), and a second one adds up the slices, multiplies T with the up matrices and rounds;
//   many rows: a first launch computes T, a second one is the shared product, whose tiles, when their K loop is done,
//              multiply their rows of T with the up matrices of the adapters that the tile has.  There T is cut
//              into 16-bit parts for the matrix instructions: three of bfloat16, or two of binary16 relative to the row's largest
//              element, so that nothing overflows; what is lost is below 2^-22 of the row's largest element.
#pragma once
#include "gemm_small_kernel.h"
#include "routed_ring.h"
#include "routed_tile.h"

namespace gemm_gfx950 {

struct AdaptersArgs {
    const void *A, *B, *down, *up;
    void *C;
    const int32_t *adapter_of;
    const float *scales;
    int64_t lda, ldb, ldc, ld_down, stride_down, ld_up, stride_up;
    int rows, N, K, adapters, rank;
    int up_kc;              // up is rank-contiguous (column-major)
    int tiles_m, tiles_n;
    Divisor by_band, by_last_rows;
    // few rows
    float *t;               // T's slices, [t_slices][rows][t_pitch]
    float *part;            // the product's, [slices][rows][part_pitch]
    int t_pitch, t_slices, t_k, turns, part_pitch, slices, k_slice;  // t_k, k_slice: k of a slice
    int down_groups;        // workgroups of the launch that compute T
    // many rows
    void *t_parts;          // [rows][parts][t_pitch], t_pitch a multiple of 64
    float *t_scale;         // [rows] powers of two that binary16 parts are to be multiplied by
};

__device__ __forceinline__ int adapter_at(const AdaptersArgs &p, int row)
{
    if (p.adapters == 0 || row >= p.rows) return -1;  // (without adapters there need not be any numbers)
    const int a = p.adapter_of[row];
    return a >= 0 && a < p.adapters ? a : -1;
}

constexpr int DOWN_ROWS = 32, DOWN_WAVES = 4;
typedef float down_part_t[DOWN_WAVES][32][33];

// ---------------------------------------------------------------------------
// Rows m0 .. m0 + 31 of A times 32 columns of a down matrix, k from k0 to k1: the waves share out the k-groups, and their sums meet in
// LDS, in wave order.  sum(r, q): row r's element of column q0 + q is handed to `take`.  KC: down is K-contiguous.
// ---------------------------------------------------------------------------
template <typename T, bool KC, typename Take>
__device__ __forceinline__ void down_block(const AdaptersArgs &p, const T *down, int row, int q0, int k0, int k1, down_part_t &part, int tid, int wave, int lane,
                                           const Take &take)
{
    constexpr int KG = Elem<T>::KG, EPL = KG / 2;
    typedef typename Frag<T>::type frag_t;
    const int q = q0 + (lane & 31) < p.rank ? q0 + (lane & 31) : p.rank - 1;
    float16_t acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
    // four groups' operands are asked for before the first is multiplied
    constexpr int AHEAD = 4;
    int k = k0 + wave * KG;
    for (; k + (AHEAD - 1) * DOWN_WAVES * KG + KG <= k1; k += AHEAD * DOWN_WAVES * KG) {
        frag_t fa[AHEAD], fb[AHEAD];
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) {
            const int kl = k + x * DOWN_WAVES * KG + (lane >> 5) * EPL;
            fa[x] = small_fragment<T, true>((const T *)p.A, p.lda, row, kl, p.K, true);
            fb[x] = small_fragment<T, KC>(down, p.ld_down, q, kl, p.K, true);
        }
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) mma(acc, fa[x], fb[x]);
    }
    for (; k < k1; k += DOWN_WAVES * KG) {
        const int kl = k + (lane >> 5) * EPL;
        const bool full = k + KG <= p.K;
        const frag_t fa = small_fragment<T, true>((const T *)p.A, p.lda, row, kl, p.K, full);
        const frag_t fb = small_fragment<T, KC>(down, p.ld_down, q, kl, p.K, full);
        mma(acc, fa, fb);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) part[wave][8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)][lane & 31] = acc[r];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = i * 8 + (tid >> 5);
        float sum = part[0][r][tid & 31];
#pragma unroll
        for (int w = 1; w < DOWN_WAVES; ++w) sum += part[w][r][tid & 31];
        take(r, tid & 31, sum);
    }
    __syncthreads();
}

// the next higher adapter number of the wave's lanes whose remainder is `turn`; 0xffffffff if there is none
__device__ __forceinline__ uint32_t next_adapter(int id, int above, uint32_t turn, uint32_t turns)
{
    return umin_over<64>(id > above && (turns == 1 || (uint32_t)id % turns == turn) ? (uint32_t)id : 0xffffffffu);
}

// ---------------------------------------------------------------------------
// Few rows: slices of T.  Workgroup `item` of down_groups: 32 rows, a slice of K, and of the adapters that the rows have those whose
// number is its turn's.
// ---------------------------------------------------------------------------
template <typename T, bool KC> __device__ __forceinline__ void down_slice(const AdaptersArgs &p, int item, down_part_t &part, int tid, int wave, int lane)
{
    const uint32_t turn = (uint32_t)item % (uint32_t)p.turns;
    const int rest = item / p.turns, slice = rest % p.t_slices, m0 = rest / p.t_slices * DOWN_ROWS;
    const int k0 = slice * p.t_k, k1 = k0 + p.t_k < p.K ? k0 + p.t_k : p.K;
    const int id = adapter_at(p, m0 + (lane & 31));
    const int row = m0 + (lane & 31) < p.rows ? m0 + (lane & 31) : p.rows - 1;
    int a = -1;
    for (;;) {
        const uint32_t next = next_adapter(id, a, turn, (uint32_t)p.turns);
        if (next == 0xffffffffu) break;
        a = __builtin_amdgcn_readfirstlane((int)next);
        const float scale = p.scales != nullptr ? p.scales[a] : 1.0f;
        const T *const down = (const T *)p.down + (int64_t)a * p.stride_down;
        for (int q0 = 0; q0 < p.rank; q0 += 32)
            down_block<T, KC>(p, down, row, q0, k0, k1, part, tid, wave, lane, [&](int r, int q, float sum) {
                if (q0 + q < p.rank && adapter_at(p, m0 + r) == a) p.t[((int64_t)slice * p.rows + m0 + r) * p.t_pitch + q0 + q] = scale * sum;
            });
    }
}

// ---------------------------------------------------------------------------
// Few rows: T and the shared product in slices of K, one launch.
// ---------------------------------------------------------------------------
template <typename T, int BM, int BN, int NST, bool BKC, bool DKC, bool DIRECT>
__global__ __launch_bounds__(256) void adapters_slices_kernel(const AdaptersArgs p)
{
    typedef TileLoop<T, BM, BN, BM / 32, 4 / (BM / 32), NST, true, BKC> Loop;
    constexpr int WM = BM / 32, WN = 4 / WM;
    union Lds { char stages[Loop::LDS_BYTES]; down_part_t part; };
    __shared__ __attribute__((aligned(1024))) Lds smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if ((int)blockIdx.x < p.down_groups) {
        down_slice<T, DKC>(p, blockIdx.x, smem.part, tid, wave, lane);
        return;
    }
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem.stages;
    // slices of a tile are neighbours, tiles of one column of them follow each other
    const int item = (int)blockIdx.x - p.down_groups, slice = item % p.slices, tile = item / p.slices;
    const int tile_n = tile / p.tiles_m, tile_m = tile - tile_n * p.tiles_m;
    const int m0 = tile_m * BM, n0 = tile_n * BN, k0 = slice * p.k_slice, k1 = k0 + p.k_slice < p.K ? k0 + p.k_slice : p.K;
    float16_t acc[Loop::FM][Loop::FN];
    Loop::zero(acc);
    if constexpr (DIRECT) {
        const int n = (k1 - k0 + Loop::BK - 1) / Loop::BK, krem = k1 - k0 - (n - 1) * Loop::BK;
        typename Loop::LoaderA la;
        typename Loop::LoaderB lb;
        la.init((const T *)p.A, p.lda, m0, p.rows, p.K, k0, wave, lane);
        lb.init((const T *)p.B, p.ldb, n0, p.N, p.K, k0, wave, lane);
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
        Loop::run(la, lb, at, n, krem, lds, acc, wave, lane);
    } else {
        granule_product<T, Loop, BM, BN, BKC>((const T *)p.A, p.lda, (const T *)p.B, p.ldb, m0, p.rows, n0, p.N, k0, k1, lds, acc, tid, wave, lane);
    }
    store_rows<float, BM, BN, WM, WN, Loop::LDS_BYTES>(acc, lds, p.part + ((int64_t)slice * p.rows + m0) * p.part_pitch + n0, p.part_pitch, p.rows - m0, p.N - n0,
                                                       wave, lane);
}

// ---------------------------------------------------------------------------
// Few rows: C from the slices.  A workgroup takes one row and JOIN_COLS columns; T's row waits in LDS, every thread has four columns.
// ---------------------------------------------------------------------------
constexpr int JOIN_COLS = 1024;
template <typename T, typename TC> __global__ __launch_bounds__(256) void adapters_join_kernel(const AdaptersArgs p)
{
    constexpr int EPC = Elem<T>::EPC;
    typedef T vec_t __attribute__((ext_vector_type(EPC)));
    typedef vec_t loose_t __attribute__((aligned(sizeof(T))));
    __shared__ float t[256];
    const int row = blockIdx.x, tid = threadIdx.x;
    const int col = (int)blockIdx.y * JOIN_COLS + tid * 4;
    const int a = adapter_at(p, row);
    if (a >= 0 && tid < p.rank) {
        float sum = p.t[(int64_t)row * p.t_pitch + tid];
        for (int s = 1; s < p.t_slices; ++s) sum += p.t[((int64_t)s * p.rows + row) * p.t_pitch + tid];
        t[tid] = sum;
    }
    float4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < p.N) {  // (a row of slices is padded to whole pieces)
        for (int s = 0; s < p.slices; ++s) acc += *(const float4_t *)(p.part + ((int64_t)s * p.rows + row) * p.part_pitch + col);
    }
    __syncthreads();
    if (col >= p.N) return;
    if (a >= 0) {
        const T *const up = (const T *)p.up + (int64_t)a * p.stride_up;
        float4_t add = {0.0f, 0.0f, 0.0f, 0.0f};
        int q = 0;
        if (p.up_kc) {
            for (; q + EPC <= p.rank; q += EPC) {
                vec_t u[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) u[c] = *(const loose_t *)(up + (int64_t)(col + c < p.N ? col + c : p.N - 1) * p.ld_up + q);
#pragma unroll
                for (int x = 0; x < EPC; ++x)
#pragma unroll
                    for (int c = 0; c < 4; ++c) add[c] = fmaf(t[q + x], (float)u[c][x], add[c]);
            }
        }
        for (; q < p.rank; ++q)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int j = col + c < p.N ? col + c : p.N - 1;
                add[c] = fmaf(t[q], (float)up[p.up_kc ? (int64_t)j * p.ld_up + q : (int64_t)q * p.ld_up + j], add[c]);
            }
        acc += add;
    }
    TC *out = (TC *)p.C + (int64_t)row * p.ldc + col;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (col + c < p.N) out[c] = rounded<TC>(acc[c]);
}

// Number of parts that an element of T is cut into
template <typename T> struct Parts;
template <> struct Parts<float> { static constexpr int N = 1; };
template <> struct Parts<_Float16> { static constexpr int N = 2; };
template <> struct Parts<__bf16> { static constexpr int N = 3; };  // (with binary32's exponents: needs no scaling)

// ---------------------------------------------------------------------------
// Many rows: the rows of adapter a among m0 .. m0 + 31 of T, full in LDS, to parts.  Eight neighbouring threads have a row.
// ---------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ void store_parts(const AdaptersArgs &p, const float *full, int pitch, int m0, int a, int tid)
{
    constexpr int NP = Parts<T>::N;
    const int r = tid / 8, g = tid % 8;
    const float scale = p.scales != nullptr ? p.scales[a] : 1.0f;
    const bool mine = adapter_at(p, m0 + r) == a;
    float factor = 1.0f;
    if constexpr (std::is_same<T, _Float16>::value) {
        float m = 0.0f;
        for (int q = g; q < p.rank; q += 8) m = fmaxf(m, fabsf(scale * full[r * pitch + q]));
#pragma unroll
        for (int s = 1; s < 8; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
        int e = 0;
        if (m > 0.0f && m < INFINITY) e = ilogbf(m);
        e = e < -126 ? -126 : e;  // (2^-e has to be a number)
        factor = ldexpf(1.0f, -e);
        if (mine && g == 0) p.t_scale[m0 + r] = ldexpf(1.0f, e);
    }
    if (!mine) return;
    T *const out = (T *)p.t_parts + (int64_t)(m0 + r) * NP * p.t_pitch;
    for (int q0 = g * 8; q0 < p.t_pitch; q0 += 64) {
        T v[NP][8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            float left = q0 + x < p.rank ? scale * full[r * pitch + q0 + x] * factor : 0.0f;
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                v[n][x] = rounded<T>(left);
                const float part = (float)v[n][x];
                left = fabsf(part) < INFINITY ? left - part : 0.0f;
            }
        }
#pragma unroll
        for (int n = 0; n < NP; ++n) {
            __builtin_memcpy(__builtin_assume_aligned(out + n * p.t_pitch + q0, 16), v[n], sizeof(v[n]));
            behind_wide_store();
        }
    }
}

// T of 32 rows, any alignment of down
template <typename T, bool KC> __global__ __launch_bounds__(DOWN_WAVES * 64) void adapters_down_any_kernel(const AdaptersArgs p)
{
    __shared__ down_part_t part;
    __shared__ float full[DOWN_ROWS * 257];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m0 = (int)blockIdx.x * DOWN_ROWS;
    const int id = adapter_at(p, m0 + (lane & 31));
    const int row = m0 + (lane & 31) < p.rows ? m0 + (lane & 31) : p.rows - 1;
    int a = -1;
    for (;;) {
        const uint32_t next = next_adapter(id, a, 0, 1);
        if (next == 0xffffffffu) break;
        a = __builtin_amdgcn_readfirstlane((int)next);
        const T *const down = (const T *)p.down + (int64_t)a * p.stride_down;
        for (int q0 = 0; q0 < p.rank; q0 += 32)
            down_block<T, KC>(p, down, row, q0, 0, p.K, part, tid, wave, lane, [&](int r, int q, float sum) { full[r * 257 + q0 + q] = sum; });
        store_parts<T>(p, full, 257, m0, a, tid);
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// T of 32 rows on direct loads: BN columns at once (rank, rounded up), NST stages of 64 k; every wave multiplies one k-group of a slab, so that
// a fragment is read from LDS once, and the waves' sums meet in LDS, in wave order.
// ---------------------------------------------------------------------------
template <typename T, int BN, int NST, bool KC> __global__ __launch_bounds__(256) void adapters_down_kernel(const AdaptersArgs p)
{
    typedef TileLoop<T, 32, BN, 1, 4, NST, true, KC> Loads;   // (its loaders and images; the multiplication is here)
    constexpr int BK = Elem<T>::BK, KG = Elem<T>::KG, EPC = Elem<T>::EPC, FN = BN / 32;
    typedef typename Frag<T>::type frag_t;
    constexpr int PITCH = BN + 1;
    constexpr int SUMS = 32 * PITCH * 4 * 4, BYTES = Loads::LDS_BYTES > SUMS ? Loads::LDS_BYTES : SUMS;
    static_assert(KGS == 4, "a k-group for each of four waves");
    __shared__ __attribute__((aligned(1024))) char smem[BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    float *const sums = (float *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m0 = (int)blockIdx.x * DOWN_ROWS;
    const int id = adapter_at(p, m0 + (lane & 31));
    const int n = (p.K + BK - 1) / BK, krem = p.K - (n - 1) * BK;
    int a = -1;
    for (;;) {
        const uint32_t next = next_adapter(id, a, 0, 1);
        if (next == 0xffffffffu) break;
        a = __builtin_amdgcn_readfirstlane((int)next);
        typename Loads::LoaderA la;
        typename Loads::LoaderB lb;
        la.init((const T *)p.A, p.lda, m0, p.rows, p.K, 0, wave, lane);
        lb.init((const T *)p.down + (int64_t)a * p.stride_down, p.ld_down, 0, p.rank, p.K, 0, wave, lane);
        auto at = [&](int h) {
            if (h > 0) {
                la.advance();
                lb.advance();
            }
            la.exact_range();
            lb.exact_range();
            if (h == n - 1 && krem < BK) {
                la.ragged_slab(krem, wave, lane);
                lb.ragged_slab(krem, wave, lane);
            }
        };
        float16_t acc[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[j][r] = 0.0f;
        const int part = krem % EPC, half = krem % KG / EPC;
        auto multiply = [&](const GEMM_LDS(char) * sA, const GEMM_LDS(char) * sB, bool last) {
            if (last && wave * KG >= krem) return;
            uint4_t mask = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
            if (last && part != 0 && wave == krem / KG && (lane >> 5) == half) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int in = part * (int)sizeof(T) - 4 * w;
                    mask[w] = in >= 4 ? 0xffffffffu : (in == 2 ? 0x0000ffffu : 0u);
                }
            }
            const frag_t fa = __builtin_bit_cast(frag_t, __builtin_bit_cast(uint4_t, fetch_group<T, 32, true>(sA, 0, wave, lane)) & mask);
            frag_t fb[FN];
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                fb[j] = fetch_group<T, BN, KC>(sB, j * 32, wave, lane);
                if (KC) fb[j] = __builtin_bit_cast(frag_t, __builtin_bit_cast(uint4_t, fb[j]) & mask);
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) mma(acc[j], fa, fb[j]);
        };
        Loads::run_with(la, lb, at, n, lds, wave, multiply);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) sums[(wave * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)) * PITCH + j * 32 + (lane & 31)] = acc[j][r];
        __syncthreads();
        for (int x = tid; x < 32 * BN; x += 256) {
            const int r = x / BN, q = x % BN;
            float s = sums[r * PITCH + q];
#pragma unroll
            for (int w = 1; w < 4; ++w) s += sums[(w * 32 + r) * PITCH + q];
            sums[r * PITCH + q] = s;  // (only this thread reads or writes it)
        }
        __syncthreads();
        store_parts<T>(p, sums, PITCH, m0, a, tid);
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// Many rows: the additions of a tile and its store, 32 rows of every wave at a time (a band): the band's accumulators leave the accumulation
// registers, which makes room for the additions', and go out as in store_rows.  lds: the K loop's, drained of loads.
// Rows of other adapters take part in a product and are not taken over: masked to zeros they would meet the adapter's matrix
// all the same, and a NaN or an infinity in it would reach them.
// ---------------------------------------------------------------------------
template <typename T, typename TC, int BM, int BN, int WM, int WN, int LDS_BYTES>
__device__ __forceinline__ void add_and_store(const AdaptersArgs &p, GEMM_LDS(char) * lds, float16_t (&acc)[BM / WM / 32][BN / WN / 32], int m0, int n0, int tid,
                                              int wave, int lane)
{
    typedef typename Frag<T>::type frag_t;
    constexpr int NT = WM * WN * 64, BK = Elem<T>::BK, KG = Elem<T>::KG, NP = Parts<T>::N;
    constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
    constexpr int BAND = WM * 32, T_BYTES = BAND * RBK, U_BYTES = BN * RBK;  // images of a band of T, of an up matrix
    constexpr int SW = TN + 8, EL = 16 / (int)sizeof(TC), LPR = TN / EL, RPI = 64 / LPR;
    constexpr int AT_T = U_BYTES, AT_IDS = AT_T + NP * T_BYTES, AT_STAGE = AT_IDS + BM * 8;
    static_assert(AT_STAGE + WM * WN * 32 * SW * 4 <= LDS_BYTES, "images and staging area");
    typedef TC vec_t __attribute__((ext_vector_type(EL)));
    typedef vec_t loose_t __attribute__((aligned(sizeof(TC))));
    GEMM_LDS(int) *ids = (GEMM_LDS(int) *)(lds + AT_IDS);
    GEMM_LDS(float) *scale = (GEMM_LDS(float) *)(lds + AT_IDS + BM * 4);
    GEMM_LDS(float) *stage = (GEMM_LDS(float) *)(lds + AT_STAGE + wave * (32 * SW * 4));
    const int wm = wave / WN, wn = wave % WN, rows = p.rows - m0, cols = p.N - n0;
    __syncthreads();  // every wave has read its last operands
    for (int r = tid; r < BM; r += NT) {
        const int a = adapter_at(p, m0 + r);
        ids[r] = a;
        scale[r] = std::is_same<T, _Float16>::value && a >= 0 ? p.t_scale[m0 + r] : 1.0f;
    }
    __syncthreads();
    int staged_a = -1, staged_q = 0;  // what the image of the up matrix holds
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        float16_t band[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            band[j] = acc[i][j];
            asm volatile("" : "+v"(band[j]));
        }
        auto band_row = [&](int x) { return x / 32 * TM + i * 32 + x % 32; };
        int a = -1;
        bool t_there = false;
        for (;;) {
            uint32_t next = 0xffffffffu;
            for (int x = lane; x < BAND; x += 64) {
                const int id = ids[band_row(x)];
                if (id > a && (uint32_t)id < next) next = (uint32_t)id;
            }
            next = umin_over<64>(next);
            if (next == 0xffffffffu) break;
            a = __builtin_amdgcn_readfirstlane((int)next);
            const T *const up = (const T *)p.up + (int64_t)a * p.stride_up;
            for (int q0 = 0; q0 < p.rank; q0 += BK) {
                if (!t_there) {
#pragma unroll 1
                    for (int n = 0; n < NP; ++n) {
                        GranuleLoader<T, BAND, NT, true> t;
                        t.fetch([&](int x) -> const T * {
                            const int row = m0 + band_row(x);
                            return row < p.rows ? (const T *)p.t_parts + ((int64_t)row * NP + n) * p.t_pitch : nullptr;
                        }, 0, p.t_pitch, q0, tid);
                        t.store(lds + AT_T + n * T_BYTES, tid);
                    }
                    t_there = p.rank <= BK;
                }
                if (staged_a != a || staged_q != q0) {
                    if (p.up_kc) {
                        GranuleLoader<T, BN, NT, true> u;
                        u.fetch([&](int c) -> const T * { return n0 + c < p.N ? up + (int64_t)(n0 + c) * p.ld_up : nullptr; }, 0, p.rank, q0, tid);
                        u.store(lds, tid);
                    } else {
                        GranuleLoader<T, BN, NT, false> u;
                        u.fetch([&](int q) -> const T * { return q < p.rank ? up + (int64_t)q * p.ld_up : nullptr; }, n0, p.N, q0, tid);
                        u.store(lds, tid);
                    }
                    staged_a = a;
                    staged_q = q0;
                }
                __syncthreads();
                float16_t add[FN];
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) add[j][r] = 0.0f;
#pragma unroll 1
                for (int kg = 0; kg < KGS && q0 + kg * KG < p.rank; ++kg) {
                    frag_t fa[NP];
#pragma unroll
                    for (int n = 0; n < NP; ++n) fa[n] = fetch_group<T, BAND, true>(lds + AT_T + n * T_BYTES, wm * 32, kg, lane);
#pragma unroll
                    for (int j = 0; j < FN; ++j) {
                        const frag_t fb = p.up_kc ? fetch_group<T, BN, true>(lds, wn * TN + j * 32, kg, lane) : fetch_group<T, BN, false>(lds, wn * TN + j * 32, kg, lane);
#pragma unroll
                        for (int n = NP - 1; n >= 0; --n) mma(add[j], fa[n], fb);  // the small parts first
                    }
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = wm * TM + i * 32 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
                    const bool mine = ids[row] == a;
                    const float f = scale[row];
#pragma unroll
                    for (int j = 0; j < FN; ++j) band[j][r] = mine ? fmaf(add[j][r], f, band[j][r]) : band[j][r];
                }
                __syncthreads();  // the images are done with
            }
        }
        // (a wave's staging area is its own)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) stage[(8 * (r >> 2) + (r & 3) + 4 * (lane >> 5)) * SW + j * 32 + (lane & 31)] = band[j][r];
        const int col = wn * TN + lane % LPR * EL;
#pragma unroll
        for (int it = 0; it < 32 / RPI; ++it) {
            const int row = wm * TM + i * 32 + it * RPI + lane / LPR;
            const GEMM_LDS(float) *src = stage + (it * RPI + lane / LPR) * SW + lane % LPR * EL;
            vec_t v;
#pragma unroll
            for (int x = 0; x < EL; ++x) v[x] = rounded<TC>(src[x]);
            if (row >= rows) continue;
            TC *dst = (TC *)p.C + (int64_t)(m0 + row) * p.ldc + n0 + col;
            if (col + EL <= cols) {
                *(loose_t *)dst = v;
                behind_wide_store();
            } else {
#pragma unroll
                for (int x = 0; x < EL; ++x)
                    if (col + x < cols) dst[x] = v[x];
            }
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

template <typename T, typename TC, int BM, int BN, bool BKC>
__global__ __launch_bounds__(256) void adapters_ring_kernel(const AdaptersArgs p)
{
    typedef RingLoop<T, BM, BN, 2, 2, true, BKC> Loop;
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tile_m, tile_n;
    if (!adapters_tile(p, tile_m, tile_n)) return;
    const int m0 = tile_m * BM, n0 = tile_n * BN;
    const int n = (p.K + Loop::BK - 1) / Loop::BK, krem = p.K - (n - 1) * Loop::BK;
    RingLoader<T, BM, 4, true> la;
    RingLoader<T, BN, 4, BKC> lb;
    la.init((const T *)p.A, p.lda, m0, p.rows, wave, lane);
    lb.init((const T *)p.B, p.ldb, n0, p.N, wave, lane);
    float16_t acc[Loop::FM][Loop::FN];
    Loop::run(la, lb, DirectLoader<T, BM, 4, true>::end_of((const T *)p.A, p.lda, p.rows, p.K), DirectLoader<T, BN, 4, BKC>::end_of((const T *)p.B, p.ldb, p.N, p.K),
              krem < Loop::BK || lb.reaches_end(n0, p.N), n, krem, lds, acc, wave, lane);
    add_and_store<T, TC, BM, BN, 2, 2, Loop::LDS_BYTES>(p, lds, acc, m0, n0, tid, wave, lane);
}

// The same through registers: any alignment, any leading dimension.
template <typename T, typename TC, int BM, int BN, bool BKC>
__global__ __launch_bounds__(256) void adapters_any_kernel(const AdaptersArgs p)
{
    typedef TileLoop<T, BM, BN, 2, 2, 4, true, BKC> Loop;  // (two stages are used: the rest is room for the additions)
    __shared__ __attribute__((aligned(1024))) char smem[Loop::LDS_BYTES];
    GEMM_LDS(char) *lds = (GEMM_LDS(char) *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tile_m, tile_n;
    if (!adapters_tile(p, tile_m, tile_n)) return;
    const int m0 = tile_m * BM, n0 = tile_n * BN;
    float16_t acc[Loop::FM][Loop::FN];
    Loop::zero(acc);
    granule_product<T, Loop, BM, BN, BKC>((const T *)p.A, p.lda, (const T *)p.B, p.ldb, m0, p.rows, n0, p.N, 0, p.K, lds, acc, tid, wave, lane);
    add_and_store<T, TC, BM, BN, 2, 2, Loop::LDS_BYTES>(p, lds, acc, m0, n0, tid, wave, lane);
}

}  // namespace gemm_gfx950
