// tree_attention_wide_bf16.hip -- osd_tree_attention of many bf16 rows.
#include "tree_attention_wide.hpp"

namespace osd {
namespace attention {

hipError_t launch_wide_bf16(const Args& args, int rows) {
    Args a = args;
    return launch_ops<Bf16Ops>(a, rows);
}

}  // namespace attention
}  // namespace osd
