// kv_attend_64.hip -- attention over 8-bit pages, head_dim 64.
#define KV_DIM 64
#include "kv_attend_launch.h"
