// latent_512.hip -- attention over 8-bit latents of 512 channels.
#define LATENT_DIM 512
#include "latent_launch.h"
