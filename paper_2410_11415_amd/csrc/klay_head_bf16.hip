// The head of a network in bf16.
#include "klay_head_launch.hip.h"

KLAY_HEAD(bf16)
