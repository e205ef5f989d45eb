// Attention over packed prompts, head dimension 64.
#include "attention_i8.h"

IPTQ_ATTENTION_I8_OF(64)
