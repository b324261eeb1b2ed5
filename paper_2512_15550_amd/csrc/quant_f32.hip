// Attention over 8-bit rows, fp32 queries and outputs
#define CTKVR_QUANT_TYPE float
#include "quant_launch.hpp"
