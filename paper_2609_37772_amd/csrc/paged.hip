// Kernels of the paged K/V cache, a code object of their own: the step's hot kernels
// keep their place in theirs (see kernels.hip).
#include "kv_internal.h"

#include "k_paged.inl"
