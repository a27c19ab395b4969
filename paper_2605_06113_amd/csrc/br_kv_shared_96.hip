// Attention of rows that are read together over the 8-bit cache, heads of 96 channels.
#include "br_kv_attend.h"

void br_kv_launch_shared_96(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st) { br_kv_attend_dim<96, BR_KV_SHARED>(p, tile, fp8, cus, st); }
