// Attention over packed prompts, head dimension 96.
#include "attention_i8.h"

IPTQ_ATTENTION_I8_OF(96)
