// The K loop of large tiles: the five-slot operand ring of gemm_tile_kernel (see there for the pipeline and what measured it) as a
// function of its loaders, so that an operand's rows can be gathered and a tile's ends are those of its group.
#pragma once
#include "routed_tile.h"

namespace gemm_gfx950 {

// Direct loads of one operand, wave w filling PER_WAVE consecutive pieces of 1 KiB of the image.
template <typename T, int R, int NW, bool KC> struct RingLoader {
    static constexpr int EPC = Elem<T>::EPC, BK = Elem<T>::BK;
    static constexpr int PER_WAVE = R * RBK / 1024 / NW;
    static_assert(PER_WAVE >= 1 && R * RBK % (1024 * NW) == 0, "tile too small for this wave count");
    static constexpr int CPR = R / EPC;
    static constexpr int ROWS_PER_LOAD = 1024 / RBK;
    int4_t rsrc;
    uint32_t off[PER_WAVE];
    int64_t step;

    static __device__ __forceinline__ int64_t granule(int64_t ld, int row0, int rmax, int i, int wave, int lane)
    {
        const int j = wave * PER_WAVE + i;
        if (KC) {
            const int r = ROWS_PER_LOAD * j + lane / GPR;
            return ((int64_t)(row0 + r < rmax ? r : rmax - 1 - row0) * ld + ((lane % GPR) ^ swz_kc(r)) * EPC) * (int64_t)sizeof(T);
        }
        const int q = 64 * j + lane, kk = q / CPR, m = ((q % CPR) ^ swz_mc<T, CPR>(kk)) * EPC;
        return ((int64_t)kk * ld + (row0 + m < rmax ? m : 0)) * (int64_t)sizeof(T);
    }
    __device__ __forceinline__ void init(const T *origin, int64_t ld, int row0, int rmax, int wave, int lane)
    {
        const uint64_t base = (uint64_t)(uintptr_t)(KC ? origin + (int64_t)row0 * ld : origin + row0);
        rsrc[0] = (int)(uint32_t)base;
        rsrc[1] = (int)(uint32_t)(base >> 32) & 0xffff;
        rsrc[2] = 0x7fffffff;
        rsrc[3] = 0x00020000;
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) off[i] = (uint32_t)granule(ld, row0, rmax, i, wave, lane);
        step = (KC ? (int64_t)BK : (int64_t)BK * ld) * (int64_t)sizeof(T);
    }
    __device__ __forceinline__ uint64_t base() const { return ((uint64_t)(uint32_t)rsrc[1] << 32) | (uint32_t)rsrc[0]; }
    // rows of the tile from `first` on are zeros (K-contiguous image)
    __device__ __forceinline__ void mask_rows(int first, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i)
            if (ROWS_PER_LOAD * (wave * PER_WAVE + i) + lane / GPR >= first) off[i] = NO_ROW;
    }
    // Whether a granule over the operand's edge can reach past its end (see DirectLoader)
    static __device__ __forceinline__ bool reaches_end(int row0, int rmax) { return !KC && rmax % EPC != 0 && row0 + R > rmax; }
    // before the loads of one of the last two slabs, of which krem k lie inside the operand: the range ends with it
    __device__ __forceinline__ void last_slab(uint64_t end, int krem, int wave, int lane)
    {
        const uint64_t left = end > base() ? end - base() : 0;
        rsrc[2] = __builtin_amdgcn_readfirstlane((left >> 31) != 0 ? 0x7fffffff : (int)(uint32_t)left);
        if (!KC) return;
#pragma unroll
        for (int i = 0; i < PER_WAVE; ++i) {
            const int r = ROWS_PER_LOAD * (wave * PER_WAVE + i) + lane / GPR;
            if (((lane % GPR) ^ swz_kc(r)) * EPC >= krem) off[i] = NO_ROW;
        }
    }
    // load number i of this wave; OFF: byte offset of the slot in the ring, wave_lds: LDS address of the wave's first piece in slot 0
    __device__ __forceinline__ void issue(uint32_t wave_lds, int slot, int i) const
    {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     : : "s"(wave_lds + (uint32_t)slot + (uint32_t)i * 1024), "v"(off[i]), "s"(rsrc) : "memory", "m0");
    }
    template <int OFF> __device__ __forceinline__ void issue_at(uint32_t wave_lds, int i) const
    {
        asm volatile("s_add_i32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds"
                     : : "s"(wave_lds), "i"(OFF + i * 1024), "v"(off[i]), "s"(rsrc) : "memory", "m0", "scc");
    }
    __device__ __forceinline__ void prefetch() {}  // what the next advance() will need
    __device__ __forceinline__ void advance(bool more)
    {
        const uint64_t to = base() + (more ? step : 0);
        rsrc[0] = (int)(uint32_t)to;
        rsrc[1] = (int)(uint32_t)(to >> 32);
    }
};

// Rows of A, gathered where there is a map (see RowsLoader)
template <typename T, int R, int NW> struct RingRowsLoader : RingLoader<T, R, NW, true> {
    typedef RingLoader<T, R, NW, true> base_t;
    uint64_t end;
    __device__ __forceinline__ void init_rows(const T *A, int64_t lda, int a_rows, const int32_t *map, int lo, int hi, int row0, int K, int wave, int lane)
    {
        typedef DirectLoader<T, R, NW, true> ends_t;
        if (map == nullptr) {
            const int there = a_rows < hi ? a_rows : hi;
            if (lo + row0 < there) {
                this->init(A + (int64_t)lo * lda, lda, row0, there - lo, wave, lane);
                end = ends_t::end_of(A + (int64_t)lo * lda, lda, there - lo, K);
                if (there < hi) this->mask_rows(there - lo - row0, wave, lane);
            } else {
                this->init(A, lda, 0, 1, wave, lane);
                end = 0;
                this->mask_rows(0, wave, lane);
            }
            return;
        }
        this->init(A, lda, 0, a_rows, wave, lane);
        end = a_rows > 0 ? ends_t::end_of(A, lda, a_rows, K) : 0;
#pragma unroll
        for (int i = 0; i < base_t::PER_WAVE; ++i) {
            const int r = base_t::ROWS_PER_LOAD * (wave * base_t::PER_WAVE + i) + lane / GPR;
            const int row = lo + row0 + r < hi ? map[lo + row0 + r] : -1;
            const uint32_t at = (uint32_t)row * (uint32_t)(lda * (int64_t)sizeof(T)) + (uint32_t)(((lane % GPR) ^ swz_kc(r)) * 16);
            this->off[i] = row >= 0 && row < a_rows ? at : NO_ROW;
        }
    }
};

// (BANDS as in TileLoop)
template <typename T, int BM, int BN, int WM, int WN, bool AKC, bool BKC, bool BANDS = false> struct RingLoop {
    static constexpr int NW = WM * WN, NT = NW * 64;
    static constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
    static constexpr int A_BYTES = BM * RBK, B_BYTES = BN * RBK, SLOT = A_BYTES > B_BYTES ? A_BYTES : B_BYTES, LDS_BYTES = NSLOT * SLOT;
    static constexpr int BK = Elem<T>::BK, KG = Elem<T>::KG, EPC = Elem<T>::EPC;
    static constexpr int NVA = A_BYTES / 1024 / NW, NVB = B_BYTES / 1024 / NW;
    typedef typename Frag<T>::type frag_t;

    // n slabs, krem k in the last one; end_a, end_b: where the operands end; checked: whether loads can reach past them.  Sets the
    // accumulators.  Ends with every load landed; waves may still be reading LDS.
    template <typename LA, typename LB>
    static __device__ __forceinline__ void run(LA &la, LB &lb, uint64_t end_a, uint64_t end_b, bool checked, int n, int krem, GEMM_LDS(char) * lds,
                                               float16_t (&acc)[FM][FN], int wave, int lane)
    {
        const int wm = wave / WN, wn = wave % WN;
        auto row_of = [&](int i) { return BANDS ? (i * WM + wm) * 32 : wm * TM + i * 32; };
        auto pin_acc = [&]() {  // in the accumulation registers at this point
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[i][j]));
        };
        auto zero_acc = [&]() {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
            pin_acc();
        };
        if (n == 0) {
            zero_acc();
            return;
        }
        // one k-group in a fixed order: block, operand fetch of the next k-group, share of the loads
        auto kgroup = [&](const frag_t(&ca)[FM], const frag_t(&cb)[FN], frag_t(&na)[FM], frag_t(&nb)[FN], const GEMM_LDS(char) * iA, const GEMM_LDS(char) * iB,
                          int kg_next, bool fetch, auto load, auto nl_tag) {
            constexpr int NL = decltype(nl_tag)::value;
            constexpr int NB = FM * FN, NF = FM + FN;
#pragma unroll
            for (int m = 0; m < NB; ++m) {
                const int mi = m / FN, mj = (mi & 1) ? FN - 1 - m % FN : m % FN;
                mma(acc[mi][mj], ca[mi], cb[mj]);
                asm volatile("" : "+a"(acc[mi][mj]));
                if (fetch) {
#pragma unroll
                    for (int f = 0; f < NF; ++f) {
                        if ((f < NB ? f : NB - 1) != m) continue;
                        if (f == 0) na[0] = Fetch<T, BM, AKC>::get(iA, row_of(0), kg_next, lane);
                        else if (f <= FN) nb[f - 1] = Fetch<T, BN, BKC>::get(iB, wn * TN + (f - 1) * 32, kg_next, lane);
                        else na[f - FN] = Fetch<T, BM, AKC>::get(iA, row_of(f - FN), kg_next, lane);
                    }
                }
                if constexpr (NL > 0) {
#pragma unroll
                    for (int q = 0; q < NL; ++q)
                        if (q * NB / NL == m) load(q);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto no_load = [](int) {};
        typedef std::integral_constant<int, 0> L0;
        const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
        const uint32_t wave_a = lds0 + wave * (NVA * 1024), wave_b = lds0 + wave * (NVB * 1024);
        constexpr bool BF = sizeof(T) == 2 && BM != 128;  // B's slab goes first
        constexpr int PA = BF ? 1 : 0, PB = 1 - PA;
        constexpr int NVX = BF ? NVB : NVA, NVY = BF ? NVA : NVB;
        auto x_issue = [&](int slot, int q) { if constexpr (BF) lb.issue(wave_b, slot, q); else la.issue(wave_a, slot, q); };
        auto y_issue = [&](int slot, int q) { if constexpr (BF) la.issue(wave_a, slot, q); else lb.issue(wave_b, slot, q); };
        auto x_advance = [&](bool more) { if constexpr (BF) lb.advance(more); else la.advance(more); };
        auto y_advance = [&](bool more) { if constexpr (BF) la.advance(more); else lb.advance(more); };
        auto a_at = [&](int h) {
            if (__builtin_expect(checked && h >= n - 2 && h < n, 0)) la.last_slab(end_a, h == n - 1 ? krem : BK, wave, lane);
        };
        auto b_at = [&](int h) {
            if (__builtin_expect(checked && h >= n - 2 && h < n, 0)) lb.last_slab(end_b, h == n - 1 ? krem : BK, wave, lane);
        };
        auto x_at = [&](int h) { if constexpr (BF) b_at(h); else a_at(h); };
        auto y_at = [&](int h) { if constexpr (BF) a_at(h); else b_at(h); };
        a_at(0);
        b_at(0);
#pragma unroll
        for (int h = 0; h < 4; ++h) {
#pragma unroll
            for (int q = 0; q < (h % 2 == 0 ? NVX : NVY); ++q) {
                if (h % 2 == 0) x_issue(h * SLOT, q);
                else y_issue(h * SLOT, q);
            }
            if (h % 2 == 0) {
                x_advance(h / 2 + 1 < n);
                x_at(h / 2 + 1);
            } else {
                y_advance(h / 2 + 1 < n);
                y_at(h / 2 + 1);
                la.prefetch();
                lb.prefetch();
            }
        }
        zero_acc();
        __builtin_amdgcn_s_waitcnt(waitcnt_vm(NVA + NVB));  // slab 0 landed
        barrier_keep_loads();
        frag_t fa[2][FM], fb[2][FN];
        {
            const GEMM_LDS(char) *cA = lds + PA * SLOT, *cB = lds + PB * SLOT;
            fa[0][0] = Fetch<T, BM, AKC>::get(cA, row_of(0), 0, lane);
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[0][j] = Fetch<T, BN, BKC>::get(cB, wn * TN + j * 32, 0, lane);
#pragma unroll
            for (int i = 1; i < FM; ++i) fa[0][i] = Fetch<T, BM, AKC>::get(cA, row_of(i), 0, lane);
        }
        auto slab_kgroups = [&](const GEMM_LDS(char) * cA, const GEMM_LDS(char) * cB, const GEMM_LDS(char) * nA, const GEMM_LDS(char) * nB, auto load_x_lo,
                                auto load_x_hi, auto load_y, const bool more, auto near_end, const int h) {
            kgroup(fa[0], fb[0], fa[1], fb[1], cA, cB, 1, true, load_x_lo, std::integral_constant<int, NVX / 2>());
            kgroup(fa[1], fb[1], fa[0], fb[0], cA, cB, 2, true, load_x_hi, std::integral_constant<int, NVX - NVX / 2>());
            x_advance(more);
            if constexpr (decltype(near_end)::value) x_at(h);
            la.prefetch();
            lb.prefetch();
            kgroup(fa[0], fb[0], fa[1], fb[1], cA, cB, 3, true, no_load, L0());
            __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(NVX));  // the next slab landed, own reads of this one done
            barrier_keep_loads();
            kgroup(fa[1], fb[1], fa[0], fb[0], nA, nB, 0, true, load_y, std::integral_constant<int, NVY>());
            y_advance(more);
            if constexpr (decltype(near_end)::value) y_at(h);
        };
        auto slab_body = [&](auto sa_tag) {
            constexpr int SA = decltype(sa_tag)::value;
            constexpr int O0 = ((SA + 0) % NSLOT) * SLOT, O1 = ((SA + 1) % NSLOT) * SLOT, O2 = ((SA + 2) % NSLOT) * SLOT, O3 = ((SA + 3) % NSLOT) * SLOT;
            constexpr int O4 = ((SA + 4) % NSLOT) * SLOT;
            auto load_x_lo = [&](int q) { if constexpr (BF) lb.template issue_at<O4>(wave_b, q); else la.template issue_at<O4>(wave_a, q); };
            auto load_x_hi = [&](int q) { if constexpr (BF) lb.template issue_at<O4>(wave_b, NVX / 2 + q); else la.template issue_at<O4>(wave_a, NVX / 2 + q); };
            auto load_y = [&](int q) { if constexpr (BF) la.template issue_at<O0>(wave_a, q); else lb.template issue_at<O0>(wave_b, q); };
            slab_kgroups(lds + (PA ? O1 : O0), lds + (PB ? O1 : O0), lds + (PA ? O3 : O2), lds + (PB ? O3 : O2), load_x_lo, load_x_hi, load_y, true,
                         std::false_type(), 0);
        };
        int t = 0;
        const int ngroup = checked ? n - 2 : n;
        for (; t + NSLOT + 2 < ngroup; t += NSLOT) {
            slab_body(std::integral_constant<int, 0>());
            slab_body(std::integral_constant<int, 2>());
            slab_body(std::integral_constant<int, 4>());
            slab_body(std::integral_constant<int, 1>());
            slab_body(std::integral_constant<int, 3>());
        }
        int sa = 0;
        auto slot = [&](int d) {
            int x = sa + d;
            x = x >= NSLOT ? x - NSLOT : x;
            return x * SLOT;
        };
        auto slab_rest = [&](auto near_end) {
            const int s0 = slot(0), spare = slot(4);
            auto load_x_lo = [&](int q) { x_issue(spare, q); };
            auto load_x_hi = [&](int q) { x_issue(spare, NVX / 2 + q); };
            auto load_y = [&](int q) { y_issue(s0, q); };
            slab_kgroups(lds + slot(PA), lds + slot(PB), lds + slot(2 + PA), lds + slot(2 + PB), load_x_lo, load_x_hi, load_y, t + 3 < n, near_end, t + 3);
            sa = sa + 2 >= NSLOT ? sa + 2 - NSLOT : sa + 2;
        };
        const int nplain = checked ? n - 5 : n - 1;
        for (; t < nplain; ++t) slab_rest(std::false_type());
        for (; t < n - 1; ++t) slab_rest(std::true_type());
        // the last slab, up to the k-group that holds the last k; what of a granule of a K-contiguous operand lies past K is masked
        const bool part = krem % EPC != 0;
        uint4_t mask = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
        if (__builtin_expect(part, 0) && (lane >> 5) == krem % KG / EPC) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int in = krem % EPC * (int)sizeof(T) - 4 * w;
                mask[w] = in >= 4 ? 0xffffffffu : (in == 2 ? 0x0000ffffu : 0u);
            }
        }
        const GEMM_LDS(char) *cA = lds + slot(PA), *cB = lds + slot(PB);
        auto last_group = [&](frag_t(&ca)[FM], frag_t(&cb)[FN], frag_t(&na)[FM], frag_t(&nb)[FN], auto kg_tag) {
            constexpr int kg = decltype(kg_tag)::value;
            if (__builtin_expect(part, 0) && kg == krem / KG) {
                if (AKC) {
#pragma unroll
                    for (int i = 0; i < FM; ++i) ca[i] = __builtin_bit_cast(frag_t, __builtin_bit_cast(uint4_t, ca[i]) & mask);
                }
                if (BKC) {
#pragma unroll
                    for (int j = 0; j < FN; ++j) cb[j] = __builtin_bit_cast(frag_t, __builtin_bit_cast(uint4_t, cb[j]) & mask);
                }
            }
            if (__builtin_expect(kg * KG < krem, 1)) kgroup(ca, cb, na, nb, cA, cB, (kg + 1) % KGS, kg + 1 < KGS, no_load, L0());
            pin_acc();
        };
        last_group(fa[0], fb[0], fa[1], fb[1], std::integral_constant<int, 0>());
        last_group(fa[1], fb[1], fa[0], fb[0], std::integral_constant<int, 1>());
        last_group(fa[0], fb[0], fa[1], fb[1], std::integral_constant<int, 2>());
        last_group(fa[1], fb[1], fa[0], fb[0], std::integral_constant<int, 3>());
        __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));  // the redundant loads past the end
    }
};

}  // namespace gemm_gfx950
