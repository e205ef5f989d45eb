// Attention over packed prompts, head dimension 32.
#include "attention_i8.h"

IPTQ_ATTENTION_I8_OF(32)
