// The head of a network in bf16.
#include "klay_head_launch.hip.h"

KLAY_HEAD_ONE(bf16)
KLAY_HEAD(bf16)
