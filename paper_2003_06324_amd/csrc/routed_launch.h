// Launchers of the grouped products, one instantiation file per kind.
#pragma once
#include "adapters_kernel.h"
#include "grouped_kernel.h"
#include "wgrad_kernel.h"

namespace gemm_gfx950 {

// forms of grouped_kernel: rows and columns of a tile; 0: through registers
enum { GROUPED_ANY = 0, GROUPED_32x128 = 1, GROUPED_64x128 = 2, GROUPED_128x128 = 3 };

template <typename T, typename TC, bool BKC> static int launch_grouped_form(int form, dim3 grid, hipStream_t s, const GroupedArgs &a)
{
    switch (form) {
    case GROUPED_32x128: return enqueue(grouped_kernel<T, TC, 32, 128, 1, 4, 4, BKC>, grid, dim3(256), s, a);
    case GROUPED_64x128: return enqueue(grouped_kernel<T, TC, 64, 128, 2, 2, 3, BKC>, grid, dim3(256), s, a);
    case GROUPED_128x128: return enqueue(grouped_kernel<T, TC, 128, 128, 2, 2, 2, BKC>, grid, dim3(256), s, a);
    default: return enqueue(grouped_any_kernel<T, TC, 64, 64, BKC>, grid, dim3(256), s, a);
    }
}
template <typename T, typename TC> int launch_grouped(int form, bool bkc, dim3 grid, hipStream_t s, const GroupedArgs &a)
{
    return bkc ? launch_grouped_form<T, TC, true>(form, grid, s, a) : launch_grouped_form<T, TC, false>(form, grid, s, a);
}

enum { WGRAD_ANY = 0, WGRAD_128x128 = 1 };
template <typename T, typename TC> int launch_wgrad(int form, dim3 grid, hipStream_t s, const WgradArgs &a)
{
    if (form == WGRAD_128x128) return enqueue(wgrad_kernel<T, TC, 128, 128, 2>, grid, dim3(256), s, a);
    return enqueue(wgrad_any_kernel<T, TC, 64, 64>, grid, dim3(256), s, a);
}

enum { ADAPTERS_ANY = 0, ADAPTERS_32x128 = 1, ADAPTERS_128x128 = 2 };
template <typename T, typename TC, bool BKC> static int launch_adapters_form(int form, dim3 grid, hipStream_t s, const AdaptersArgs &a)
{
    switch (form) {
    case ADAPTERS_32x128: return enqueue(adapters_kernel<T, TC, 32, 128, 1, 4, 4, BKC>, grid, dim3(256), s, a);
    case ADAPTERS_128x128: return enqueue(adapters_kernel<T, TC, 128, 128, 2, 2, 2, BKC>, grid, dim3(256), s, a);
    default: return enqueue(adapters_any_kernel<T, TC, 64, 64, BKC>, grid, dim3(256), s, a);
    }
}
template <typename T, typename TC> int launch_adapters(int form, bool bkc, dim3 grid, hipStream_t s, const AdaptersArgs &a)
{
    return bkc ? launch_adapters_form<T, TC, true>(form, grid, s, a) : launch_adapters_form<T, TC, false>(form, grid, s, a);
}
template <typename T> int launch_adapters_down(bool kc, dim3 grid, hipStream_t s, const AdaptersArgs &a)
{
    return kc ? enqueue(adapters_down_kernel<T, true>, grid, dim3(256), s, a) : enqueue(adapters_down_kernel<T, false>, grid, dim3(256), s, a);
}

#define ROUTED_FORMS(PREFIX, T, TC)                                                                        \
    PREFIX template int launch_grouped<T, TC>(int, bool, dim3, hipStream_t, const GroupedArgs &);           \
    PREFIX template int launch_wgrad<T, TC>(int, dim3, hipStream_t, const WgradArgs &);                     \
    PREFIX template int launch_adapters<T, TC>(int, bool, dim3, hipStream_t, const AdaptersArgs &);

}  // namespace gemm_gfx950
