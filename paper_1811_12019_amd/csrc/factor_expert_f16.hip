// The experts' factors from f16 rows.
#define KFAC_EXPERT_KIND 1
#include "factor_expert.h"
