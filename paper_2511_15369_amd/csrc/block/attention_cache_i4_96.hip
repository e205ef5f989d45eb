// Attention over the 4-bit cache, head dimension 96.
#include "attention_cache_i4.h"

IPTQ_ATTENTION_CACHE_I4_OF(96)
