// Scales for blocks of 8-bit pools, and page tables, a code object of their own.
#include "kv_internal.h"

#include <algorithm>

#include "k_paged_blocks.inl"
