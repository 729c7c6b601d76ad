// expanded_128.hip -- attention in the expanded form, keys of 128 channels beside the rotary ones.
#define EXPANDED_NOPE 128
#include "expanded_launch.h"
