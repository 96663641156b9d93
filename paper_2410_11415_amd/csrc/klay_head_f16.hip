// The head of a network in f16.
#include "klay_head_launch.hip.h"

KLAY_HEAD_ONE(f16)
KLAY_HEAD(f16)
