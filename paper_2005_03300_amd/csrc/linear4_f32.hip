#include "linear4.h"

namespace gcn {

template <> int linear4_of<float>(const TileArgs& a, const Weights4& w, hipStream_t s) { return w.gated ? linear4_impl<float, true>(a, w, s) : linear4_impl<float, false>(a, w, s); }

}  // namespace gcn
