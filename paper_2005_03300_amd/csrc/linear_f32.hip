// The products of a linear layer on 32-bit elements.
#define GCN_LINEAR_ELEM float
#include "linear_launch.h"
