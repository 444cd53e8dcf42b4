// The tree attention's split pass for bf16 queries.
#include "tree_dev.h"

namespace dwkv {

void launch_tree_split_bf16(const TreeArgs& a, hipStream_t s) { launch_tree_split<true>(a, s); }

}  // namespace dwkv
