// kv_attend_128.hip -- attention over 8-bit pages, head_dim 128.
#define KV_DIM 128
#include "kv_attend_launch.h"
