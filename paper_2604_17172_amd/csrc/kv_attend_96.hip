// kv_attend_96.hip -- attention over 8-bit pages, head_dim 96.
#define KV_DIM 96
#include "kv_attend_launch.h"
