// The host side of libpwlq in one translation unit: the search, quantizer and inner product with their kernels, and the
// entry points of the operators around them, which share its error text.  Those operators' kernels are sources of their own.
#include "../pwlq_api.hip"

#include "calls.h"
