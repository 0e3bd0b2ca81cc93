// Attention of many new rows over the paged K/V cache, a code object of its own.
#include "kv_internal.h"

#include "k_paged_prompt.inl"
