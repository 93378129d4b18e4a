// Which tiles a product takes, and its launch, for one element type.
#pragma once
#include "linear_tile.h"

namespace gcn {

template <typename T, int LIES>
static bool whole_pieces(const void* p, int64_t ld, int64_t along) {
    constexpr int E = Elem<T>::E;
    return ((uintptr_t)p & 15) == 0 && ld % E == 0 && (LIES == BY_K || along % E == 0);
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
    const size_t lds = 2 * (BM + BN) * 128;
    if (whole_pieces<T, LA>(a.A, a.lda, a.M) && whole_pieces<T, LB>(a.B, a.ldb, a.N))
        launch_lds<k_linear_tile<T, BM, BN, WM, WN, LA, LB, true>>(grid, WM * WN * 64, lds, s, a);
    else
        launch_lds<k_linear_tile<T, BM, BN, WM, WN, LA, LB, false>>(grid, WM * WN * 64, lds, s, a);
    GCN_LAUNCH_CHECK();
    if (splits > 1) {
        const int64_t threads = a.M * ((a.N + 3) / 4);
        hipLaunchKernelGGL((k_linear_join<T>), dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, splits);
        GCN_LAUNCH_CHECK();
    }
    return GCN_OK;
}

template <typename T, int LA, int LB>
static int linear_product(const TileArgs& a, hipStream_t s) {
    const int64_t cus = device_info().cus;
    auto tiles = [&](int b) { return ((a.M + b - 1) / b) * ((a.N + b - 1) / b); };
    if (tiles(256) >= cus * 3 / 4) return launch_tile<T, 256, 256, 2, 4, LA, LB>(a, 1, s);
    const int64_t stages = (a.K + 8 * Elem<T>::E - 1) / (8 * Elem<T>::E);
    if (tiles(128) >= cus * 3 / 4) return launch_tile<T, 128, 128, 2, 2, LA, LB>(a, 1, s);
    const int64_t most = (stages + 3) / 4, want = (2 * cus + tiles(64) - 1) / tiles(64);
    const int64_t splits = want < most ? want : most;
    return launch_tile<T, 64, 64, 2, 2, LA, LB>(a, (int)(splits < 1 ? 1 : splits > 1024 ? 1024 : splits), s);
}

template <> int linear_forward_of<GCN_LINEAR_ELEM>(const TileArgs& a, hipStream_t s) { return linear_product<GCN_LINEAR_ELEM, BY_K, BY_MN>(a, s); }
template <> int linear_dx_of<GCN_LINEAR_ELEM>(const TileArgs& a, hipStream_t s) { return linear_product<GCN_LINEAR_ELEM, BY_K, BY_K>(a, s); }
template <> int linear_dw_of<GCN_LINEAR_ELEM>(const TileArgs& a, hipStream_t s) { return linear_product<GCN_LINEAR_ELEM, BY_MN, BY_MN>(a, s); }

}  // namespace gcn
