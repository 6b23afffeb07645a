// The experts' factors from f32 rows.
#define KFAC_EXPERT_KIND 2
#include "factor_expert.h"
