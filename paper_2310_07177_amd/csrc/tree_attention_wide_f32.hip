// tree_attention_wide_f32.hip -- osd_tree_attention of many fp32 rows.
#include "tree_attention_wide.hpp"

namespace osd {
namespace attention {

hipError_t launch_wide_f32(const Args& args, int rows) {
    Args a = args;
    return launch_ops<F32Ops>(a, rows);
}

}  // namespace attention
}  // namespace osd
