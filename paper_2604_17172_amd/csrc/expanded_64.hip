// expanded_64.hip -- attention in the expanded form, keys of 64 channels beside the rotary ones.
#define EXPANDED_NOPE 64
#include "expanded_launch.h"
