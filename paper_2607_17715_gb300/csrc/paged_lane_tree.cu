// Paged attention of few query rows in fp32 contexts, trees of tokens (c2kv_paged_attend_tree).
#define C2KV_TREES
#include "paged_lane.cu"
