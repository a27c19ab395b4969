// Attention over the 8-bit cache, heads of 256 channels.
#include "br_kv_attend.h"

void br_kv_launch_attend_256(const BrKvAttend &p, int tile, bool fp8, int cus, hipStream_t st) { br_kv_attend_dim<256>(p, tile, fp8, cus, st); }
