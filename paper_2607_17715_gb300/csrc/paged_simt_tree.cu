// Paged attention of fp32 contexts, trees of tokens (c2kv_paged_attend_tree).
#define C2KV_TREES
#include "paged_simt.cu"
