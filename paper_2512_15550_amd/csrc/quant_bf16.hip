// Attention over 8-bit rows, bf16 queries and outputs
#define CTKVR_QUANT_TYPE bf16_t
#include "quant_launch.hpp"
