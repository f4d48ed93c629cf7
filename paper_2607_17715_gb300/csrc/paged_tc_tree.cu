// Paged attention of many query rows, trees of tokens (c2kv_paged_attend_tree).
#define C2KV_TREES
#include "paged_tc.cu"
