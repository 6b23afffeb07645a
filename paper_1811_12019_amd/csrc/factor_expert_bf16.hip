// The experts' factors from bf16 rows.
#define KFAC_EXPERT_KIND 0
#include "factor_expert.h"
