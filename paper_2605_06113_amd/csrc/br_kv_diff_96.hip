// Differential attention over the 8-bit cache, heads of two times 48 channels.
#include "br_kv_attend.h"

void br_kv_launch_diff_96(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st) { br_kv_attend_dim<96, BR_KV_DIFF>(p, tile, fp8, cus, st); }
