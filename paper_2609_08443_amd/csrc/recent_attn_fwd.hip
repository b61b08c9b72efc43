// Forward pass of the attention over recent histories (recent_attn_rows.h).
#include "recent_attn_rows.h"

namespace sa {
namespace attn {

hipError_t launch_rows_fwd(const RowsArgs& f, bool bf16, int32_t d, bool wide, hipStream_t stream) {
    return launch_rows<false>(f, bf16, d, wide, stream);
}

template <typename T, int D, bool WIDE, bool BWD>
RowsShape shape_of() {
    using C = RowsCfg<T, D, WIDE, BWD>;
    return {C::BQ, C::UNIT, C::PER_CU};
}
template <bool WIDE, bool BWD>
RowsShape shape_of(bool bf16, int32_t d) {
    if (bf16) return d == 64 ? shape_of<uint16_t, 64, WIDE, BWD>() : shape_of<uint16_t, 128, WIDE, BWD>();
    return d == 64 ? shape_of<float, 64, WIDE, BWD>() : shape_of<float, 128, WIDE, BWD>();
}
RowsShape rows_shape(bool bf16, int32_t d, bool wide, bool bwd) {
    if (wide) return bwd ? shape_of<true, true>(bf16, d) : shape_of<true, false>(bf16, d);
    return bwd ? shape_of<false, true>(bf16, d) : shape_of<false, false>(bf16, d);
}

}  // namespace attn
}  // namespace sa
