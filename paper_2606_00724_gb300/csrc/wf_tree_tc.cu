// The tensor-core attention over shared prompts, compiled for caches in pages
// (wf_tree_attn).
#define WF_TREE
#include "wf_prefix_tc.cu"
