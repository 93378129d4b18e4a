// Which tiles a product takes, and its launch, for one element type.
#pragma once
#include "launch_rules.h"
#include "linear_few.h"
#include "linear_thirds.h"
#include "linear_tile.h"

namespace gcn {

template <typename T, int LIES>
static bool whole_pieces(const void* p, int64_t ld, int64_t along) {
    constexpr int E = Elem<T>::E;
    return ((uintptr_t)p & 15) == 0 && ld % E == 0 && (LIES == BY_K || along % E == 0);
}

template <typename T>
static int launch_join(const TileArgs& a, int splits, hipStream_t s) {
    const int64_t threads = a.M * ((a.N + Elem<T>::E - 1) / Elem<T>::E);
    if (splits > 8) hipLaunchKernelGGL((k_linear_join<T, 16>), dim3((unsigned)((threads + 63) / 64)), dim3(1024), 0, s, a, splits);
    else hipLaunchKernelGGL((k_linear_join<T, 1>), dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, splits);
    GCN_LAUNCH_CHECK();
    return GCN_OK;
}

template <typename T, int BM, int BN, int WM, int WN, int LA, int LB>
static int launch_tile(TileArgs a, int splits, hipStream_t s) {
    const int64_t tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
    if (tm * tn * (WM * WN * 64) > UINT32_MAX) return fail(GCN_ERR_RANGE, "linear: more results than one launch has threads for");
    constexpr int BK = 8 * Elem<T>::E;
    a.tiles_m = (int32_t)tm;
    a.tiles_n = (int32_t)tn;
    const int64_t stages = (a.K + BK - 1) / BK;
    a.k_share = (stages + splits - 1) / splits * BK;
    splits = (int)((a.K + a.k_share - 1) / a.k_share);
    ScratchLease lease;
    if (splits > 1) {
        void* p = nullptr;
        GCN_TRY(lease.get(&p, (size_t)splits * a.M * a.N * 4, s));
        a.part = (float*)p;
    }
    const dim3 grid((unsigned)(tm * tn), (unsigned)splits);
    if constexpr (sizeof(T) == 4) {
        hipLaunchKernelGGL((k_linear_thirds<BM, BN, WM, WN, LA, LB>), grid, dim3(WM * WN * 64), 0, s, a);
    } else {
        if (whole_pieces<T, LA>(a.A, a.lda, a.M) && whole_pieces<T, LB>(a.B, a.ldb, a.N))
            hipLaunchKernelGGL((k_linear_tile<T, BM, BN, WM, WN, LA, LB, true>), grid, dim3(WM * WN * 64), 0, s, a);
        else
            hipLaunchKernelGGL((k_linear_tile<T, BM, BN, WM, WN, LA, LB, false>), grid, dim3(WM * WN * 64), 0, s, a);
    }
    GCN_LAUNCH_CHECK();
    if (splits > 1) return launch_join<T>(a, splits, s);
    return GCN_OK;
}

template <typename T, int LA, int LB>
static int linear_product(const TileArgs& a, hipStream_t s) {
    const bool direct = whole_pieces<T, LA>(a.A, a.lda, a.M) && whole_pieces<T, LB>(a.B, a.ldb, a.N);
    const TileChoice c = choose_tiles(a.M, a.N, a.K, sizeof(T) == 4, sizeof(T) == 2 && direct, device_info().cus);
    if constexpr (sizeof(T) == 2)
        if (c.edge == 256) return launch_tile<T, 256, 256, 2, 4, LA, LB>(a, c.splits, s);
    if (c.edge == 128) return launch_tile<T, 128, 128, 2, 2, LA, LB>(a, c.splits, s);
    return launch_tile<T, 64, 64, 2, 2, LA, LB>(a, c.splits, s);
}

template <typename T, int C, int RT>
static int launch_few(TileArgs a, hipStream_t s) {
    constexpr int STEP = 4 * Elem<T>::E * FEW_WAVES;              // values of k that a workgroup takes at a time
    const int strips = (a.N + 16 * C - 1) / (16 * C);
    // One launch where the strips give enough compute units work; else up to 128 workgroups, each with two steps at least.  (16 rows in bf16, k of 16384, with up to 64, 128
    // and 256 workgroups: 64 columns 9.0, 9.1, 9.0 us, 256 columns 14.5, 11.7, 9.8, 512 columns 24.2, 15.5, 12.3; k of 4096 and less 0 to 13 % between 64 and 128.)
    int64_t splits = 1;
    if (strips < FEW_STRIPS) {
        splits = 128 / strips;
        const int64_t most = (a.K + 2 * STEP - 1) / (2 * STEP);
        if (splits > most) splits = most;
    }
    const int64_t steps = (a.K + STEP - 1) / STEP;
    a.k_share = (steps + splits - 1) / splits * STEP;
    splits = (a.K + a.k_share - 1) / a.k_share;
    ScratchLease lease;
    if (splits > 1) {
        void* p = nullptr;
        GCN_TRY(lease.get(&p, (size_t)splits * a.M * a.N * 4, s));
        a.part = (float*)p;
    }
    launch_lds<k_linear_few<T, C, RT>>(dim3((unsigned)((strips + 7) / 8 * 8), (unsigned)splits), FEW_WAVES * 64, few_lds<T, C, RT>(), s, a, strips);
    GCN_LAUNCH_CHECK();
    return splits > 1 ? launch_join<T>(a, (int)splits, s) : GCN_OK;
}

template <typename T>
static int linear_forward_impl(const TileArgs& a, hipStream_t s) {
    const int64_t cus = device_info().cus;
    // Two fragments of 16 rows are what k_linear_few holds.  17 and 32 rows there and as tiles of 64, bf16: 1024 x 4096 4.9 and 5.5 us against 9.1 and 10.0, 256 x 1024 3.7 and 3.8 against
    // 4.3, 4096 x 4096 13.8 and 15.7 against 13.6 and 14.6; fp32 21.6 and 23.8 against 31.  Tiles are the faster for long sums over few columns (16384 x 1024 in bf16 13.8 us
    // against 40).
    if (a.M > 32) return linear_product<T, BY_K, BY_MN>(a, s);
    // the widest strips that are still one for every compute unit
    const int c = a.N >= 64 * cus ? 4 : a.N >= 32 * cus ? 2 : 1;
    if (a.M <= 16) return c == 4 ? launch_few<T, 4, 1>(a, s) : c == 2 ? launch_few<T, 2, 1>(a, s) : launch_few<T, 1, 1>(a, s);
    return c == 4 ? launch_few<T, 4, 2>(a, s) : c == 2 ? launch_few<T, 2, 2>(a, s) : launch_few<T, 1, 2>(a, s);
}

template <> int linear_forward_of<GCN_LINEAR_ELEM>(const TileArgs& a, hipStream_t s) { return linear_forward_impl<GCN_LINEAR_ELEM>(a, s); }
template <> int linear_dx_of<GCN_LINEAR_ELEM>(const TileArgs& a, hipStream_t s) { return linear_product<GCN_LINEAR_ELEM, BY_K, BY_K>(a, s); }
template <> int linear_dw_of<GCN_LINEAR_ELEM>(const TileArgs& a, hipStream_t s) { return linear_product<GCN_LINEAR_ELEM, BY_MN, BY_MN>(a, s); }

}  // namespace gcn
