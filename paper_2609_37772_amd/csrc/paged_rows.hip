// Attention of new rows over the paged K/V cache, a code object of its own.
#include "kv_internal.h"

#include <algorithm>

#include "k_paged_rows.inl"
