// Attention over packed prompts, head dimension 128.
#include "attention_i8.h"

IPTQ_ATTENTION_I8_OF(128)
