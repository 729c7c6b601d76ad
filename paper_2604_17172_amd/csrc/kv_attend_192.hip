// kv_attend_192.hip -- attention over 8-bit pages, head_dim 192.
#define KV_DIM 192
#include "kv_attend_launch.h"
