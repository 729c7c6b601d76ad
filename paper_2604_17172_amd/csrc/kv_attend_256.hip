// kv_attend_256.hip -- attention over 8-bit pages, head_dim 256.
#define KV_DIM 256
#include "kv_attend_launch.h"
