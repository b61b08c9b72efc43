// The queries' gradients of the attention over recent histories (recent_attn_rows.h).
#include "recent_attn_rows.h"

namespace sa {
namespace attn {

hipError_t launch_rows_dq(const RowsArgs& f, bool bf16, int32_t d, bool wide, hipStream_t stream) {
    return launch_rows<true>(f, bf16, d, wide, stream);
}

}  // namespace attn
}  // namespace sa
