// The products of a linear layer on half-precision elements.
#define GCN_LINEAR_ELEM _Float16
#include "linear_launch.h"
