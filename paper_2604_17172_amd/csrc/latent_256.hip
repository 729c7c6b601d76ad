// latent_256.hip -- attention over 8-bit latents of 256 channels.
#define LATENT_DIM 256
#include "latent_launch.h"
