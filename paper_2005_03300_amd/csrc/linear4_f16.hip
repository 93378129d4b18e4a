#include "linear4.h"

namespace gcn {

template <> int linear4_of<_Float16>(const TileArgs& a, const Weights4& w, hipStream_t s) { return w.gated ? linear4_impl<_Float16, true>(a, w, s) : linear4_impl<_Float16, false>(a, w, s); }

}  // namespace gcn
