// The products of a linear layer on bfloat16 elements.
#define GCN_LINEAR_ELEM __bf16
#include "linear_launch.h"
