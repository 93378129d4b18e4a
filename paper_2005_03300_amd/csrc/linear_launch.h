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
        const int64_t threads = a.M * ((a.N + Elem<T>::E - 1) / Elem<T>::E);
        hipLaunchKernelGGL((k_linear_join<T>), dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, splits);
        GCN_LAUNCH_CHECK();
    }
    return GCN_OK;
}

// The tiles of a product: their edge, and in how many shares the sum over k is cut.
struct TileChoice {
    int edge, splits;
};
// The choice with the least estimated time.  A compute unit works through its tiles at a share of the matrix units' rate that grows with the edge (measured on
// 16384 x 4096 x 4096 in bf16: 1.16 PFLOP/s at 256, 1.03 at 128, 0.70 at 64; in fp32 the three are alike), with a single small tile at a time at little more
// than half of that; splits fill the chip where there are few tiles, and cost partial results written and read again and a launch.
inline TileChoice choose_tiles(int64_t M, int64_t N, int64_t K, bool fp32, int64_t cus) {
    const double rate = fp32 ? 0.59e6 : 4.5e6;                    // FLOP per microsecond of one compute unit
    const int64_t depth = fp32 ? 32 : 64, stages = (K + depth - 1) / depth;
    TileChoice best{64, 1};
    double least = 1e300;
    for (const int edge : {256, 128, 64}) {
        if (fp32 && edge == 256) continue;                        // (nothing to win, and fewer tiles)
        const int64_t tiles = ((M + edge - 1) / edge) * ((N + edge - 1) / edge);
        for (int64_t splits = 1; splits <= 512; splits += splits < 4 ? 1 : splits / 2) {
            const int64_t share = (stages + splits - 1) / splits;
            if (splits > 1 && (share < 4 || tiles * (splits - 1) > 4 * cus)) break;
            const int64_t count = tiles * splits, rounds = (count + cus - 1) / cus;
            const double full = fp32 ? 1.0 : edge == 256 ? 1.0 : edge == 128 ? 0.9 : 0.62;
            const double part = edge == 256 || rounds >= (edge == 128 ? 2 : 4) ? full : 0.55 * full;
            double us = rounds * (2.0 * edge * edge * depth * share / (rate * part) + 1.0);
            if (splits > 1) us += 3.0 + splits * (double)M * N * 8 / 4.0e6;
            if (us < least) {
                least = us;
                best = {edge, (int)splits};
            }
        }
    }
    return best;
}

template <typename T, int LA, int LB>
static int linear_product(const TileArgs& a, hipStream_t s) {
    const TileChoice c = choose_tiles(a.M, a.N, a.K, sizeof(T) == 4, device_info().cus);
    if constexpr (sizeof(T) == 2)
        if (c.edge == 256) return launch_tile<T, 256, 256, 2, 4, LA, LB>(a, c.splits, s);
    if (c.edge == 128) return launch_tile<T, 128, 128, 2, 2, LA, LB>(a, c.splits, s);
    return launch_tile<T, 64, 64, 2, 2, LA, LB>(a, c.splits, s);
}

template <> int linear_forward_of<GCN_LINEAR_ELEM>(const TileArgs& a, hipStream_t s) { return linear_product<GCN_LINEAR_ELEM, BY_K, BY_MN>(a, s); }
template <> int linear_dx_of<GCN_LINEAR_ELEM>(const TileArgs& a, hipStream_t s) { return linear_product<GCN_LINEAR_ELEM, BY_K, BY_K>(a, s); }
template <> int linear_dw_of<GCN_LINEAR_ELEM>(const TileArgs& a, hipStream_t s) { return linear_product<GCN_LINEAR_ELEM, BY_MN, BY_MN>(a, s); }

}  // namespace gcn
